// The body of the attention kernels over a latent cache (tree_attention_latent.hip), for LatentParams args and constants DL, DR (channels), NT
// (loads that leave no copy in the caches) and RG: groups of 16 query rows of a chunk, 4; or 1, for calls of no more rows, where two of the
// scores' wavefronts have nothing to do but to meet the others.  (Text and not a function: inlined as one, the compiler's code for 64 rows
// took up to 6 % longer.)
    const LatentParams &p = args;
    constexpr int SR = RG == 4 ? 2 : 1;                                    // ... of a wavefront of scores
    using C = Cfg<DL, DR>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int G = p.workgroups;
    // Neighbours in the order of the work share an L2: the hardware deals workgroups to the eight dies in turn.
    const int w = (G & 7) == 0 ? ((int)blockIdx.x & 7) * (G >> 3) + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
    const int tree_tiles = (p.n + KEYS - 1) / KEYS;
    // ---- this workgroup's piece of the work.  Lengths and places of 64 sequences, one per lane (in most calls all of them: one trip to
    // memory).
    int b_lanes = 0, len_l = 0;
    int64_t base_l = 0;
    auto fetch = [&](int b0) __attribute__((always_inline)) {
        b_lanes = b0;
        len_l = -1;
        if (b0 + lane < p.B) {
            len_l = min(max(p.lens[b0 + lane], 0), p.max_prefix);
            base_l = p.seq_base[b0 + lane];
        }
    };
    const bool uncut = !p.header;                                          // one workgroup for every unit: nothing to plan
    if (!uncut) fetch(0);
    auto tiles_at = [&](int b0) __attribute__((always_inline)) {           // of sequence b0 + lane
        if (b0 != b_lanes) fetch(b0);
        return len_l >= 0 ? tree_tiles + (int)(((unsigned)len_l + KEYS - 1) / KEYS) : 0;
    };
    int total = 0, most = 0;
    for (int b0 = 0; b0 < p.B && !uncut; b0 += 64) {
        const int t = tiles_at(b0);
        total += wave_last(wave_scan(t));
        most = max(most, wave_max(t));
    }
    // A unit of t tiles in pieces of s: s turns, and t / s parts to fold, each counted as a quarter of a turn; s = sqrt(t) / 2 is the least of
    // both together.  (One sequence of 16384 keys, 16 heads, one node: 32 us, with pieces down to four tiles 55; 8192 keys, 128 heads: 33
    // and 41.  Where there are more units, equal shares are longer than that.)
    const int pairs = p.B * p.chunks, least = max(MIN_TILES, (int)(0.5f * __builtin_amdgcn_sqrtf((float)most)));
    // Pieces that stay within a sequence, all of a unit's alike, may be up to CROSS tiles longer than equal shares of everything, whose pieces
    // can go on in the next unit: queries and output twice.  (8 sequences of 100..3000 keys x 32 heads x 14 nodes: 32 us, without the
    // allowance 37; 24 of 100..1500 x 8 heads x 44 nodes: 41 and 44.  It loses where shares are short: 1024 keys x 128 heads x 44 nodes, 17
    // tiles where the share is 12: 40.1 and 38.5.  An allowance of 24: 4096 keys x 128 heads x 44 nodes 84 us, with 12 or none 76.)
    int per = max((int)(((int64_t)total * p.chunks + G - 1) / G), least), aligned = 0;
    if (pairs <= G && !uncut) {
        if (per >= most) {
            aligned = per;
        } else {
            auto fits = [&](int size) {
                int sum = 0;
                for (int b0 = 0; b0 < p.B; b0 += 64) sum += wave_last(wave_scan(small_div(tiles_at(b0) + size - 1, size)));
                return sum * p.chunks <= G;
            };
            int lo = per, hi = per + CROSS;
            if (fits(hi)) {
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (fits(mid)) hi = mid;
                    else lo = mid + 1;
                }
                aligned = hi;
            }
        }
    }
    // Else as many teams as the chunks leave room for, one workgroup for every chunk, that go through all sequences' tiles in step: a tile
    // is read from memory once for all of its chunks then, and from the L2 by the others.  (Equal pieces of everything, where that would
    // leave too many workgroups without work, each at a place of its own: the ragged batch of 16 sequences of 512 to 4096 keys, 15 chunks
    // each, took 150 us, at 7 TB/s from behind the L2.)  That is worth up to a quarter more tiles than equal pieces have: never in step, 2 x
    // 16384 keys x 64 heads x 120 nodes took 560 us instead of 513 and 6 x 300..9000 keys x 16 heads x 120 nodes 172 instead of 144; always,
    // 4096 keys x 128 heads x 44 nodes 83 instead of 76 and 4 x 500..2000 keys 111 instead of 104.
    bool in_step = false;
    if (!aligned && !uncut && p.chunks <= G) {
        const int teams = G / p.chunks, of_team = max((total + teams - 1) / teams, least);
        in_step = (int64_t)of_team * 4 <= (int64_t)per * 5;
        if (in_step) per = of_team;
    }
    // b, chunk: where the piece begins; tile: its first tile there; left: its tiles in all
    int b = -1, chunk = 0, tile = 0, left = 0, n_pieces = 1, number = 0, each = 0;
    if (uncut) {
        b = small_div(w, p.chunks);
        chunk = w - b * p.chunks;
        left = 0x7fffffff;
        aligned = 1;
        fetch(b & ~63);
    } else if (aligned) {
        int before = 0;
        for (int b0 = 0; b0 < p.B && b < 0; b0 += 64) {
            const int t = tiles_at(b0), e = small_div(t + aligned - 1, aligned), s = wave_scan(e * p.chunks);
            const int last = before + s;
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(w < last);
            if (beyond) {
                const int l = __builtin_ctzll(beyond);
                b = b0 + l;
                n_pieces = __builtin_amdgcn_readlane(e, l);
                const int tiles = __builtin_amdgcn_readlane(t, l), k = w - (__builtin_amdgcn_readlane(last, l) - n_pieces * p.chunks);
                number = k / p.chunks;                               // (the same keys of all chunks next to each other)
                chunk = k - number * p.chunks;
                each = (tiles + n_pieces - 1) / n_pieces;
                tile = number * each;
                left = min(each, tiles - tile);
            }
            before = __builtin_amdgcn_readlane(last, 63);
        }
    } else {
        const int64_t all = (int64_t)total * (in_step ? 1 : p.chunks), from = (int64_t)(in_step ? w / p.chunks : w) * per;
        const int each_seq = in_step ? 1 : p.chunks;
        int64_t before = 0;
        left = (int)max((int64_t)0, min((int64_t)per, all - from));
        for (int b0 = 0; b0 < p.B && b < 0 && left > 0; b0 += 64) {
            const int t = tiles_at(b0), s = wave_scan(t);
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(from < before + (int64_t)s * each_seq);
            if (beyond) {
                const int l = __builtin_ctzll(beyond);
                b = b0 + l;
                const int tiles = __builtin_amdgcn_readlane(t, l);
                const int k = (int)(from - (before + (int64_t)(__builtin_amdgcn_readlane(s, l) - tiles) * each_seq));
                chunk = in_step ? w % p.chunks : k / tiles;
                tile = in_step ? k : k - chunk * tiles;
            }
            before += (int64_t)__builtin_amdgcn_readlane(s, 63) * each_seq;
        }
    }
    if (b < 0 || left <= 0) {
        if (tid == 0 && pairs > G) p.header[w].pieces = 0;
        return;
    }

    // ---- places of this lane
    const bool scorer = wave < 4;                                          // S^T and weights, else O^T
    const int part = wave & 3, rh = part & 1, kg = part >> 1;              // a scorer's rows 32 rh .. and keys 16 kg ..; else the channels DL / 4 part ..
    const int krow = 16 * kg + col;
    const int k_at = krow * 128 + ((grp ^ swz(krow)) << 4);                // panel's chunk grp; the other half of a panel: ^ 64
    const int k_half = C::PANELS * C::PANEL + krow * 64 + ((grp ^ swz_half(krow)) << 4);
    const int pw_at = C::P_AT + (32 * rh + col) * 64 + (((2 * kg + (grp >> 1)) ^ swz_half(col)) << 4) + (grp & 1) * 8;       // weights written; + 16 rows * 64
    const int pr_at = C::P_AT + col * 64 + ((grp ^ swz_half(col)) << 4);   // weights read
    const int jr = col >> 2, v_row = 8 * grp + jr;                         // of the 16 lanes of a transpose load: row (+ 4 for the second load), 4 channels
    const int v_at = v_row * 128 + ((((col & 3) >> 1) ^ swz(v_row)) << 4) + (col & 1) * 8 + part * (DL / 4) * (2 * KEYS);
    // Tile loads, by those of O^T: 8 rows of a panel per instruction.
    const int lrow = 8 * part + (lane >> 3);
    const uint32_t load_at = (uint32_t)(lrow * C::ROWB + (((lane & 7) ^ swz(lrow)) << 4));
    const int hrow = 16 * (part & 1) + (lane >> 2);                        // (half panels: 16 rows, two wavefronts bring the same)
    const uint32_t load_half = (uint32_t)(hrow * C::ROWB + C::PANELS * 128 + (((lane & 3) ^ swz_half(hrow)) << 4));

    for (bool begun = false;; begun = true) {
        b = uniform(b);
        chunk = uniform(chunk);
        tile = uniform(tile);
        left = uniform(left);
        if (b >= b_lanes + 64) fetch(b & ~63);
        const int len = __builtin_amdgcn_readlane(len_l, b - b_lanes), tiles = tree_tiles + (int)(((unsigned)len + KEYS - 1) / KEYS);
        const int from = tile, count = min(left, tiles - tile);
        const bool whole = from == 0 && count == tiles, first = from == 0, last = from + count == tiles;
        const int slot = aligned ? 2 * w : 2 * w + (begun ? 1 : 0);

        if (scorer) {
            // Query operands: rows col + 16 rg of this half of the chunk (behind the last: that one), channels 32 ks + 8 grp .. + 7.  They come by
            // way of the places of tiles 2 and 3, whole cache lines, once for both wavefronts that
            // share them (each by itself, 16 rows an instruction and half a line of each, waited 11500 cycles for them: 16 heads under 14 nodes and 128
            // keys 18.5 us instead of 15.9, 16 x 512..4096 keys under 60 nodes 115 instead of 108).
            // And which tree nodes the rows see among this lane's 4 keys: 4 bits per row and tree tile.
            bf16x8_t q[SR][C::KS];
            uint64_t bits[2][2];
            if constexpr (SR == 1) bits[1][0] = bits[1][1] = 0;
            unsigned char *const queries = lds + 2 * C::TILE;
            auto query_row = [&](int row, int &i) __attribute__((always_inline)) {                 // of the chunk: its place, its node
                const int r = min(chunk * ROWS + row, p.rows - 1), h = row_div(r, p.by_nrows);
                i = p.row0 + r - h * (p.n - p.row0);
                return (const unsigned char *)(p.q + (((int64_t)b * p.H + h) * p.node_stride + i) * C::D);
            };
#pragma unroll
            for (int half = 0; half < 2 && (RG == 4 || wave == 0); ++half) {      // 8 rows of a panel per instruction
                const int row = 16 * wave + 8 * half + (lane >> 3);
                int i;
                const unsigned char *src = query_row(row, i) + (((lane & 7) ^ swz(row & 15)) << 4);
#pragma unroll
                for (int x = 0; x < C::PANELS + (DR == 64); ++x) load_to_lds16_at(src + x * 128, queries + x * 2 * C::PANEL + (16 * wave + 8 * half) * 128);
            }
            if (DR == 32 && (RG == 4 || wave == 0)) {
                const int row = 16 * wave + (lane >> 2);
                int i;
                const unsigned char *src = query_row(row, i) + C::PANELS * 128 + (((lane & 3) ^ swz_half(row & 15)) << 4);
                load_to_lds16_at(src, queries + C::PANELS * 2 * C::PANEL + 16 * wave * 64);
            }
#pragma unroll
            for (int rg = 0; rg < SR; ++rg) {
                int i;
                query_row(32 * rh + 16 * rg + col, i);
                const uint64_t *row = p.mask_bits + (int64_t)i * p.mask_words;
                bits[rg][0] = row[0];
                bits[rg][1] = tree_tiles > 2 ? row[1] : 0;
            }
            MCSD_WAIT_VMCNT(0);
            meet();                                                        // the queries are here
            if (RG == 1 && rh == 1) {                                      // no rows: their flags, and every meeting
                auto grown = [&](int t) __attribute__((always_inline)) {
                    const u32x4_t flags = *(const u32x4_t *)(lds + C::FLAG_AT + (t & 1) * 16);
                    return (uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) & GROWN) != 0;
                };
                auto meet3 = [&]() __attribute__((always_inline)) {
                    meet();
                    meet();
                    meet();
                };
                if (lane < 2) *(int *)(lds + C::FLAG_AT + lane * 16 + 4 * wave) = 0;
                meet();
                for (int t = 0; t < count; ++t) {
                    if (t > 0 && grown(t - 1)) meet3();
                    meet();
                }
                if (grown(count - 1)) meet3();
                meet();
            } else {
#pragma unroll
            for (int rg = 0; rg < SR; ++rg)
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    const int row = 32 * rh + 16 * rg + col;
                    q[rg][ks] = *(const bf16x8_t *)(queries + (DR == 32 && ks == C::KS - 1 ? C::PANELS * 2 * C::PANEL + row * 64 + ((grp ^ swz_half(col)) << 4)
                                                                                            : (ks >> 1) * 2 * C::PANEL + row * 128 + (((grp + 4 * (ks & 1)) ^ swz(col)) << 4)));
                }
            unsigned seen = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) seen |= (unsigned)((bits[k & 1][k >> 2] >> (32 * (k >> 1 & 1) + 16 * kg + 4 * grp)) & 15) << (4 * k);      // tile k / 2, rows k % 2
            float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, start[2] = {0.f, 0.f};      // (start: minus the reference, 0 while no key has been seen)
            f32x4_t s[SR];
            // Weights are rounded to bf16, which is what the product with the values takes: half a step, 2^-8 of each, and as they are off
            // independently of each other, of an output made from many keys less (0.0017 to 0.0023 of it in all, of which its own rounding is
            // 0.0017).  Their sum is of the weights in fp32.
            auto weigh = [&](int t, float (&sum)[2]) __attribute__((always_inline)) {
                unsigned char *pw = lds + pw_at + (t & 1) * C::P_BYTES;
#pragma unroll
                for (int rg = 0; rg < SR; ++rg) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = fast_exp2(fmaf(s[rg][i], p.c, start[rg]));
                    sum[rg] = (e[0] + e[1]) + (e[2] + e[3]);
                    const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[0], (__bf16)e[1]}),
                                        __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[2], (__bf16)e[3]})};
                    *(u32x2_t *)(pw + rg * 16 * 64) = pk;
                }
            };
            float sum[2] = {0.f, 0.f};                                     // of the last tile's weights
            // Of tile t, whose scores s holds: its maxima over all keys, new references, its weights again; what O^T has of the tiles before is
            // multiplied by alpha.
            auto outgrown = [&](int t) __attribute__((always_inline)) {
#pragma unroll
                for (int rg = 0; rg < SR; ++rg) {
                    const float m = row_max(max4(s[rg]) * p.c);
                    if (grp == 0) *(float *)(lds + C::MAX_AT + (kg * ROWS + 32 * rh + 16 * rg + col) * 4) = m;
                }
                meet();
#pragma unroll
                for (int rg = 0; rg < SR; ++rg) {
                    const int row = 32 * rh + 16 * rg + col;
                    const float m = fmaxf(*(const float *)(lds + C::MAX_AT + row * 4), *(const float *)(lds + C::MAX_AT + (ROWS + row) * 4));
                    const float now = m > ref[rg] + SLACK ? m : ref[rg];
                    const float alpha = now == ref[rg] ? 1.f : fast_exp2(ref[rg] - now);
                    ref[rg] = now;
                    start[rg] = now == -INFINITY ? 0.f : -now;
                    l[rg] *= alpha;
                    if (kg == 0 && grp == 0) *(float *)(lds + C::ALPHA_AT + row * 4) = alpha;
                }
                weigh(t, sum);
                meet();
                meet();                                                    // (O^T uses the other place for weights until then)
            };
            auto flagged = [&](int t) __attribute__((always_inline)) { return *(const u32x4_t *)(lds + C::FLAG_AT + (t & 1) * 16); };
            meet();                                                        // the first tile is here
            for (int t = 0; t < count; ++t) {
                const int at = from + t, st = (t & 3) * C::TILE, k0 = anew(k_at) + st;
                auto key_of = [&](int ks) __attribute__((always_inline)) {
                    return *(const bf16x8_t *)(lds + (DR == 32 && ks == C::KS - 1 ? k_half + st : (k0 ^ ((ks & 1) << 6)) + (ks >> 1) * C::PANEL));
                };
                const u32x4_t flags = flagged(t - 1);                      // (looked at behind the products)
                f32x4_t n[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};             // (of the two row groups, or of every other step)
                constexpr int AHEAD = 8;                                   // steps that key operands are read ahead
                bf16x8_t kf[AHEAD];
#pragma unroll
                for (int ks = 0; ks < AHEAD; ++ks) kf[ks] = key_of(ks);
                asm volatile("s_nop 1" : "+v"(n[0]), "+v"(n[1]));          // (two wait states from a vector instruction to a product that reads its result)
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int rg = 0; rg < SR; ++rg) mfma(n[SR == 2 ? rg : ks & 1], kf[ks % AHEAD], q[rg][ks]);
                    if (ks + AHEAD < C::KS) kf[ks % AHEAD] = key_of(ks + AHEAD);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (t > 0 && __builtin_expect((uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) & GROWN) != 0, 0)) outgrown(t - 1);
                settle();
#pragma unroll
                for (int rg = 0; rg < SR; ++rg) {
                    asm volatile("" : "+v"(n[rg]));
                    if constexpr (SR == 2) {
                        s[rg] = n[rg];
                    } else {
                        asm volatile("" : "+v"(n[1]));
                        s[rg] = n[0] + n[1];
                    }
                    l[rg] += sum[rg];
                }
                const bool tree = at < tree_tiles;
                const int here = tree ? KEYS : len - (at - tree_tiles) * KEYS;
                bool wrong = false;
                if (tree || here < KEYS) {
                    unsigned bits;
                    if (tree) {
                        bits = seen >> (8 * at);
#pragma unroll
                        for (int rg = 0; rg < SR; ++rg)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                s[rg][i] += s[rg][i] - s[rg][i];           // (infinities as well are NaN)
                                wrong |= s[rg][i] != s[rg][i];
                            }
                    } else {
                        const int mine = min(max(here - 16 * kg - 4 * grp, 0), 4);
                        bits = ((1u << mine) - 1) * 0x11u;
                    }
#pragma unroll
                    for (int rg = 0; rg < SR; ++rg)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[rg][i] = (bits >> (4 * rg + i)) & 1 ? s[rg][i] : -INFINITY;
                }
                weigh(t, sum);
                bool grow = false;
#pragma unroll
                for (int rg = 0; rg < SR; ++rg) grow |= max4(s[rg]) * p.c > ref[rg] + SLACK;
                const int flag = (__builtin_amdgcn_ballot_w64(grow) != 0 ? GROWN : 0) | (__builtin_amdgcn_ballot_w64(wrong) != 0 ? WRONG : 0);
                if (lane == 0) *(int *)(lds + C::FLAG_AT + (t & 1) * 16 + 4 * wave) = flag;
                __builtin_amdgcn_s_setprio(0);
                meet();
            }
            {
                const u32x4_t flags = flagged(count - 1);
                if (__builtin_expect((uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) & GROWN) != 0, 0)) outgrown(count - 1);
                l[0] += sum[0];
                if constexpr (SR == 2) l[1] += sum[1];
            }
            // sums and references of the rows, while O^T takes the last tile
#pragma unroll
            for (int rg = 0; rg < SR; ++rg) {
                const float sum = row_sum(l[rg]);
                const int row = 32 * rh + 16 * rg + col;
                if (grp == 0) *(float *)(lds + C::MAX_AT + (kg * ROWS + row) * 4) = sum;
                if (kg == 0 && grp == 0) *(float *)(lds + C::ALPHA_AT + row * 4) = ref[rg];
            }
            meet();
            }
        } else {
            const int64_t base = (int64_t)__builtin_amdgcn_readlane((int)(base_l >> 32), b - b_lanes) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)base_l, b - b_lanes);
            const unsigned char *past = uniform((const unsigned char *)(p.cache + base));
            const unsigned char *nodes = uniform((const unsigned char *)(p.tree + (int64_t)b * p.node_stride * C::D));
            auto request = [&](int t) __attribute__((always_inline)) {     // tile t of this part, LOADS loads
                const int at = from + t, here = at < tree_tiles ? p.n - at * KEYS : len - (at - tree_tiles) * KEYS;      // keys of the tile (or more)
                const unsigned char *src = at < tree_tiles ? nodes + (int64_t)at * C::TILE : past + (int64_t)(at - tree_tiles) * C::TILE;
                unsigned char *dst = lds + (t & 3) * C::TILE + 8 * part * 128;
                const int row = anew(lrow);
                if (here >= KEYS) {
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x) load_to_lds16<NT>(src + x * 128, load_at, dst + x * C::PANEL);
                    if constexpr (DR == 32) load_to_lds16<NT>(src, load_half, lds + (t & 3) * C::TILE + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                } else {                                                   // rows behind the last: zeros
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x)
                        load_to_lds16_at(row < here ? src + x * 128 + load_at : no_row + (anew(lane) & 7) * 16, dst + x * C::PANEL);
                    if constexpr (DR == 32)
                        load_to_lds16_at(hrow < here ? src + load_half : no_row + (lane & 3) * 16, lds + (t & 3) * C::TILE + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                }
            };
            f32x4_t o[RG][C::CB];
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) o[rg][cb] = (f32x4_t){0, 0, 0, 0};
            request(0);
            if (count > 1) request(1);
            meet();                                                        // the queries are here
            if (count > 1) MCSD_WAIT_VMCNT(C::LOADS);
            else MCSD_WAIT_VMCNT(0);
            meet();                                                        // the first tile is here
            // In turn t, while the scores of tile t are made, tile t - 1 is added up, tile t + 2 requested into the place of tile t - 2, and
            // behind it tile t + 1 is here.
            if (count > 2) request(2);
            if (count > 2) MCSD_WAIT_VMCNT(C::LOADS);
            else MCSD_WAIT_VMCNT(0);
            meet();
            for (int t = 1;; ++t) {
                const int vb = anew(v_at) + ((t - 1) & 3) * C::TILE, pb = anew(pr_at) + ((t - 1) & 1) * C::P_BYTES;
                auto value_of = [&](int cb) __attribute__((always_inline)) {
                    const int a = vb ^ ((cb & 3) << 5), at = (cb >> 2) * C::PANEL;
                    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + a + at));
                    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + (a ^ 48) + at + 512));
                    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                };
                const u32x4_t flags = *(const u32x4_t *)(lds + C::FLAG_AT + ((t - 1) & 1) * 16);
                constexpr int AHEAD = C::CB;                               // value operands read ahead
                bf16x8_t pf[RG], vf[AHEAD];
#pragma unroll
                for (int rg = 0; rg < RG; ++rg) pf[rg] = *(const bf16x8_t *)(lds + pb + rg * 16 * 64);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < AHEAD; ++cb) vf[cb] = value_of(cb);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (RG == 4) asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(pf[2]), "+v"(pf[3]));       // (one wait for weights and flags)
                else asm volatile("" : "+v"(pf[0]));
                const int flag = uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])), on = flag & GROWN;
                if (__builtin_expect((flag & WRONG) != 0, 0)) {
                    clear_wrong(lds + ((t - 1) & 3) * C::TILE + part * (DL / 4) * (2 * KEYS), lane, DL / 4 * (2 * KEYS));
#pragma unroll
                    for (int cb = 0; cb < AHEAD; ++cb) vf[cb] = value_of(cb);
                }
                if (__builtin_expect(on != 0, 0)) {                        // a reference was outgrown by that tile
                    meet();
                    meet();
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg) pf[rg] = *(const bf16x8_t *)(lds + pb + rg * 16 * 64);
                }
                const int own = lds_at(lds + C::P_AT) + (t & 1) * C::P_BYTES + part * 1024 + anew(lane) * 16;      // (weights that are done with)
                const int alpha = lds_at(lds + C::ALPHA_AT) + anew(col) * 4;
                multiply(t > 1 ? on : 0, o, alpha, own);                   // (before that it is zero)
                if (on) meet();
                const int next = t + 2, at = from + next, here = at < tree_tiles ? p.n - at * KEYS : len - (at - tree_tiles) * KEYS;
                const unsigned char *src = at < tree_tiles ? nodes + (int64_t)at * C::TILE : past + (int64_t)(at - tree_tiles) * C::TILE;
                unsigned char *dst = lds + (next & 3) * C::TILE;
                int ask = uniform(next < count && here >= KEYS ? 1 : 0);
                asm volatile("" : "+s"(ask));
                if (next < count && !ask) request(next);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) {
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg) mfma(o[rg][cb], vf[cb % AHEAD], pf[rg]);
                    if (cb + AHEAD < C::CB) vf[cb % AHEAD] = value_of(cb + AHEAD);
                    // (a load takes as long as the products of a block)
                    load_if<NT>(ask, src + cb * 128, load_at, dst + 8 * part * 128 + cb * C::PANEL);
                    if (cb == C::CB - 1) {
                        if constexpr (DR == 64) load_if<NT>(ask, src + C::PANELS * 128, load_at, dst + 8 * part * 128 + C::PANELS * C::PANEL);
                        else load_if<NT>(ask, src, load_half, dst + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (next < count) MCSD_WAIT_VMCNT(C::LOADS);
                else MCSD_WAIT_VMCNT(0);
                meet();
                if (t == count) break;
            }
            // ---- the rows' output, or this part of it: 16 rows x 128 bytes at a time by way of LDS (where weights were), so that a store
            // writes whole cache lines (8 bytes a lane from the registers, 32 a row, took 8200 cycles: 2 x 128 heads under 14 nodes and 192 keys 16.1 us
            // instead of 14.9).
#pragma unroll
            for (int rg = 0; rg < RG; ++rg) {
                settle();
                __builtin_amdgcn_sched_barrier(0);
                if (chunk * ROWS + 16 * rg >= p.rows) break;
                unsigned char *const own = lds + C::P_AT + part * 2048;
                const int at = anew(lane), own_row = at >> 3, own_at = own_row * 128 + (((at & 7) ^ own_row) << 4);
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) asm volatile("" : "+v"(o[rg][cb]));
                const int c = at & 15, g = at >> 4, row = 16 * rg + c;
                const float sum = *(const float *)(lds + C::MAX_AT + row * 4) + *(const float *)(lds + C::MAX_AT + (ROWS + row) * 4);
                const float ref = *(const float *)(lds + C::ALPHA_AT + row * 4);
                unsigned char *dst[2];                                     // of rows own_row and own_row + 8
                bool there[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int row = 16 * rg + 8 * half + own_row, r = chunk * ROWS + row;
                    there[half] = r < p.rows;
                    if (whole) {
                        const int h = row_div(r, p.by_nrows), i = p.row0 + r - h * (p.n - p.row0);
                        dst[half] = (unsigned char *)(p.out + (((int64_t)b * p.H + h) * p.node_stride + i) * DL + part * (DL / 4) + (at & 7) * 8);
                    } else {
                        dst[half] = (unsigned char *)(p.part_o + ((int64_t)slot * p.slot_rows + row) * DL + part * (DL / 4) + (at & 7) * 4);
                    }
                }
                auto store = [&](int x) __attribute__((always_inline)) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const u32x4_t v = *(const u32x4_t *)(own + own_at + half * 1024);
                        if (there[half]) *(u32x4_t *)(dst[half] + x * 128) = v;
                    }
                };
                unsigned char *const to = own + c * 128;
                if (whole) {
                    const float inv = 1.f / sum;
#pragma unroll
                    for (int x = 0; x < C::CB / 4; ++x) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x4_t y = o[rg][4 * x + k] * inv;
                            const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[0], (__bf16)y[1]}),
                                                __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[2], (__bf16)y[3]})};
                            *(u32x2_t *)(to + (((2 * k + (g >> 1)) ^ (c & 7)) << 4) + (g & 1) * 8) = pk;
                        }
                        store(x);
                    }
                } else {
                    if (part == 0 && g == 0 && chunk * ROWS + row < p.rows) {
                        const int64_t of = (int64_t)slot * p.slot_rows + row;
                        p.part_m[of] = ref;
                        p.part_l[of] = sum;
                    }
#pragma unroll
                    for (int x = 0; x < C::CB / 2; ++x) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) *(f32x4_t *)(to + (((4 * k + g) ^ (c & 7)) << 4)) = o[rg][2 * x + k];
                        store(x);
                    }
                }
            }
        }
        left -= count;
        const bool more = !aligned && left > 0;
        // What to fold: one word for every unit where no more of them than workgroups, else for every piece (only the last unit that begins
        // in it can go on in others).
        if (p.header && tid == 0 && (pairs <= G ? first : !more)) {
            LatentHeader h = {};
            if (first && !last) {                                          // it begins here: who goes on with it
                h.b = b;
                h.chunk = chunk;
                h.first = slot;
                h.stride = aligned || in_step ? 2 * p.chunks : 2;
                h.second = 2 * w + h.stride;
                h.pieces = aligned ? n_pieces : 1 + (tiles - count + per - 1) / per;
            }
            p.header[pairs <= G ? b * p.chunks + chunk : w] = h;
        }
        if (!more) return;
        tile = 0;
        if (in_step) {
            ++b;
        } else if (++chunk == p.chunks) {
            chunk = 0;
            ++b;
        }
    }
