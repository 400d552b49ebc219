// Work split of a wave over a cache held in 4 bits (part of wpp_plan_tiles).
#include <algorithm>
#include <cstdint>
#include <cstring>
#include <utility>
#include <vector>

#include "../../include/wpp.h"
#include "wpp_host.h"
#include "wpp_plan_format.h"

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The kernel for few rows: CTAs that an SM holds, of blocks of at most 8 rows and of more; what a unit costs besides its key steps, in
// steps; and the fewest steps that a block is cut for.
constexpr int kFewCtas = 3, kFewCtasWide = 2;
constexpr int64_t kUnitSteps = 3, kLeastSteps = 2;
// Which kernel takes a chunk, if a wave has both: the one for few rows walks its keys once per block, and has a walk done in a quarter
// of what a tile's takes.  Attention call in a graph, us, tiles | few rows: 4 walks a tile, 8 x 8 tokens over 4,096 (64/8 heads of 128)
// 56 | 52; 5 walks, 32 x 10 over 2,048 102 | 132; 6 walks of 5 tiles, 16 x 18 over 4,000 (40/8) 424 | 137.
constexpr int64_t kFewWalks = 4;
// A wave has both, tiles alone or few rows alone, by the estimated time of each: a start, and for what falls to a CTA a time per key
// step, of few rows with kUnitSteps a unit, of tiles with one half and with both (heads of 64: 0.7 of either).  Estimated and measured:
// 64 x 1 over 255..16,383 (64/8) 130, 128; 16 x 32 over 2,000 (32/8) tiles 50, 48, few rows 99, 101; 64 x 5 over 1,000 (32/8) 92, 102 and
// 59, 65; 1 x 64 over 1,024 (8/2 of 64) 18, 22 and 9, 9.7; 12 x 1..300 over 0..700 (8/2 of 64) tiles 24, 24, both 34, 30.
constexpr double kFewStart = 3.0, kFewStep = 1.45, kTileStart = 7.0, kTileStep1 = 2.7, kTileStep2 = 3.2, kCombine = 4.0;
constexpr int64_t kFewShort = 4;
// Tiles: fewest key steps of a part, and rounds of tiles up to which the longest come first.  The parts of a wave are of equal length,
// whatever the tiles': against equal numbers of parts, us, 4 x 76..106 tokens over 0..18,257 (32/8) 193 -> 104, 4 x 47..191 over 0..31,067
// (64/8) 435 -> 332; cut for any win, 2 x 183..211 over 0..1,065 (32/8) would take 28 where whole tiles take 25.
constexpr int64_t kTileLeastSteps = 4, kTileLeastWin = 3;
constexpr int64_t kTileOrderRounds = 16;

// Row blocks of the kernel for few rows: heads of a KV group, and tokens, WPP_FEW_ROWS rows at most.
static int32_t few_heads(int32_t group) { return std::min<int32_t>(group, WPP_FEW_ROWS); }
static int32_t few_tokens(int32_t group) { return std::max<int32_t>(1, WPP_FEW_ROWS / few_heads(group)); }

static int64_t few_blocks(const wpp_batch_desc* d, int64_t C) {
    const int32_t G = d->num_q_heads / d->num_kv_heads, h = few_heads(G), t = few_tokens(G);
    return (C + t - 1) / t * ((G + h - 1) / h) * d->num_kv_heads;
}

// Tiles of two halves of 128 rows: two heads of a KV group over the same rows where the group is even (both then end at the same key),
// else two row blocks of a head; blocks of at most 64 rows take several heads in a half (see WppUnit).  Of a block of `rows` rows:
// places for heads in a half, and heads of a tile.
static int32_t tile_rows(int32_t G) { return G % 2 == 0 ? WPP_HALF_M : 2 * WPP_HALF_M; }
static void tile_heads(int32_t G, int32_t rows, int32_t* pack, int32_t* per_tile) {
    *pack = *per_tile = 1;
    if (rows > WPP_HALF_M) return;
    while (*pack < 8 && G % (2 * *pack) == 0 && WPP_HALF_M / (2 * *pack) >= rows) *pack *= 2;
    int32_t whole = 1;
    while (whole < G) whole *= 2;
    *per_tile = G % (2 * *pack) == 0 ? 2 * *pack : *pack;
    if (*pack < whole && whole <= 8 && WPP_HALF_M / whole >= rows) {
        *pack = whole;
        *per_tile = G;
    }
}
static int64_t tiles_of(const wpp_batch_desc* d, int64_t C) {
    const int32_t G = d->num_q_heads / d->num_kv_heads, block = tile_rows(G);
    int32_t pack, per_tile;
    tile_heads(G, block, &pack, &per_tile);
    int64_t n = C / block * (d->num_q_heads / per_tile);
    if (C % block == 0) return n;
    tile_heads(G, (int32_t)(C % block), &pack, &per_tile);
    return n + d->num_q_heads / per_tile;
}

// Key steps of a tile's parts, at most: the least with which the parts of fewer tiles than CTAs are no more than those; of more tiles, a
// CTA's share of all steps, which cuts what alone would take longer; but no tile is cut where that wins less than kTileLeastWin steps.
// `tiles`: (how many, of so many steps).  Tiles that fill the CTAs are cut only into as many parts as `slots` hold: a wave that needs
// no scratch uncut is not refused for its cuts by the entry point that has the built-in array alone.
static int64_t tile_part_steps(const std::vector<std::pair<int64_t, int64_t>>& tiles, int64_t ctas, int64_t slots) {
    int64_t n = 0, all = 0, longest = 1;
    for (const auto& t : tiles) {
        n += t.first;
        all += t.first * t.second;
        longest = std::max(longest, t.second);
    }
    int64_t lo = std::min<int64_t>(std::max<int64_t>(kTileLeastSteps, (all + ctas - 1) / ctas), longest), hi = longest;
    while (n < ctas && lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        int64_t parts = 0;
        for (const auto& t : tiles) parts += t.first * ((t.second + mid - 1) / mid);
        if (parts <= ctas) hi = mid;
        else lo = mid + 1;
    }
    int64_t parts = 0;
    for (const auto& t : tiles) parts += t.second > lo ? t.first * ((t.second + lo - 1) / lo) : 0;
    return longest - lo >= kTileLeastWin && (n < ctas || parts <= slots) ? lo : longest;
}

static int64_t scratch_slots(const wpp_batch_desc* d) {
    return (int64_t)((wpp_static_scratch_bytes() - WPP_WS_HEADER_BYTES) / (2 * WPP_HALF_M * (d->head_dim + 1) * sizeof(float)));
}

// Whether the kernel for few rows has a chunk: walks per tile 0, kFewWalks or any number.
static bool is_few(const wpp_batch_desc* d, int64_t C, int64_t walks) {
    return walks == INT64_MAX || few_blocks(d, C) <= walks * tiles_of(d, C);
}
static int64_t few_walks(const wpp_batch_desc* d, const wpp_plan_opts* o, const int32_t* prefix_lens, const int32_t* chunk_lens) {
    if (o->shape) return o->shape == 1 ? 0 : INT64_MAX;
    const int32_t G = d->num_q_heads / d->num_kv_heads;
    const int64_t choices[3] = {kFewWalks, INT64_MAX, 0};
    const double narrow = d->head_dim == 64 ? 0.7 : 1.0;
    double best_us = 0.0;
    int64_t best = kFewWalks;
    for (int64_t walks : choices) {
        double few = 0.0, steps = 0.0, least = 0.0;
        int64_t rows = 0, num_tiles = 0, longest = 0;
        std::vector<std::pair<int64_t, int64_t>> tiles;
        bool both_halves = false;
        double few_longest = 0.0;
        for (int i = 0; i < d->num_requests; ++i) {
            const int64_t C = chunk_lens[i], end = (prefix_lens[i] + C + WPP_TILE_N - 1) / WPP_TILE_N;
            if (C == 0) continue;
            if (is_few(d, C, walks)) {
                few += (double)few_blocks(d, C) * (double)(end + kUnitSteps);
                rows = std::max(rows, std::min<int64_t>(C, few_tokens(G)) * few_heads(G));
                least = std::max(least, (double)std::min(end + kUnitSteps, kFewShort));
                few_longest = std::max(few_longest, (double)(end + kUnitSteps));
            } else {
                const int64_t n = tiles_of(d, C);
                tiles.emplace_back(n, end);
                num_tiles += n;
                steps += (double)n * (double)end;
                longest = std::max(longest, end);
                int32_t pack, per_tile;
                tile_heads(G, (int32_t)std::min<int64_t>(C, tile_rows(G)), &pack, &per_tile);
                both_halves |= per_tile > pack || C > WPP_HALF_M;
            }
        }
        double us = 0.0;
        if (few > 0.0) {
            const double share = few / ((double)(rows <= 8 ? kFewCtas : kFewCtasWide) * o->max_ctas);
            us += kFewStart + kFewStep * narrow * std::max(share, least) + (few_longest > share && few_longest > (double)kFewShort + kUnitSteps ? kCombine : 0.0);
        }
        if (num_tiles > 0) {
            const double part = (double)tile_part_steps(tiles, o->max_ctas, scratch_slots(d));
            us += kTileStart + (both_halves ? kTileStep2 : kTileStep1) * narrow *
                                   (num_tiles < o->max_ctas ? part : steps / o->max_ctas + part / 2);
            if (part < (double)longest) us += kCombine;
        }
        if (walks == kFewWalks || us < best_us) { best = walks; best_us = us; }
    }
    return best;
}

size_t wpp_kv4_plan_bytes(const wpp_batch_desc* d, const wpp_plan_opts* o, int64_t T) {
    const int32_t G = d->num_q_heads / d->num_kv_heads, h = few_heads(G), t = few_tokens(G);
    const int64_t base = (T / t + d->num_requests) * ((G + h - 1) / h) * d->num_kv_heads;
    const int64_t units = o->force_kv_splits >= 2 ? base * o->force_kv_splits : base + kFewCtas * (int64_t)o->max_ctas;
    size_t n = sizeof(WppPlanHeader) + 2 * align_up(sizeof(int32_t) * (size_t)(d->num_requests + 1), 16);
    n += sizeof(WppUnit) * (size_t)units + align_up(sizeof(int32_t) * ((size_t)std::max(units, kFewCtas * (int64_t)o->max_ctas) + 1), 16);
    n += sizeof(WppCombine) * (size_t)(T * d->num_q_heads / t + (int64_t)d->num_requests * d->num_q_heads);
    const int64_t tiles = (T / WPP_HALF_M + d->num_requests) * d->num_q_heads;
    n += sizeof(WppUnit) * (size_t)(o->force_kv_splits >= 2 ? tiles * o->force_kv_splits : tiles + (int64_t)o->max_ctas);
    n += sizeof(WppCombine) * (size_t)tiles;
    return align_up(n, 256);
}

int wpp_kv4_plan(const wpp_batch_desc* d, const wpp_plan_opts* o, const int32_t* prefix_lens, const int32_t* chunk_lens, int64_t T,
                 int64_t pairs, void* plan_host, size_t plan_host_bytes, wpp_plan_info* info) {
    const int R = d->num_requests, Hq = d->num_q_heads, Hkv = d->num_kv_heads, G = Hq / Hkv;
    if (plan_host_bytes < wpp_kv4_plan_bytes(d, o, T)) return WPP_ERR_PLAN_MISMATCH;
    auto steps_for = [](int64_t keys) { return (int32_t)((keys + WPP_TILE_N - 1) / WPP_TILE_N); };

    const int32_t heads = few_heads(G), toks = few_tokens(G);
    const int64_t walks = few_walks(d, o, prefix_lens, chunk_lens);
    // The CTAs take equal shares of the blocks' key steps, in order: a block is cut where a share ends.
    int64_t n_base = 0, all_steps = 0;
    int32_t max_rows = 0;
    for (int i = 0; i < R; ++i) {
        if (!is_few(d, chunk_lens[i], walks)) continue;
        n_base += few_blocks(d, chunk_lens[i]);
        for (int64_t r0 = 0; r0 < chunk_lens[i]; r0 += toks) {
            const int32_t rows = (int32_t)std::min<int64_t>(toks, chunk_lens[i] - r0);
            all_steps += steps_for(prefix_lens[i] + r0 + rows) * (int64_t)((G + heads - 1) / heads) * Hkv;
            max_rows = std::max(max_rows, rows * heads);
        }
    }
    if (n_base > 0x3fffffff) return WPP_ERR_INVALID_ARG;
    const int64_t most_ctas = (int64_t)(max_rows <= 8 ? kFewCtas : kFewCtasWide) * o->max_ctas;
    int64_t share = std::max<int64_t>((all_steps + kUnitSteps * (n_base + most_ctas) + most_ctas - 1) / most_ctas, kUnitSteps + kLeastSteps);
    // Where the part that begins at key step `at` ends: a CTA takes what is left of its share, no less than kLeastSteps, and the rest too
    // if that is little.  next: it is the next CTA's.
    auto part_end = [&](int32_t steps, int32_t at, int64_t& left, bool& next) {
        next = left < kUnitSteps + kLeastSteps && left < share;
        if (next) left = share;
        int32_t n = (int32_t)std::min<int64_t>(steps - at, std::max<int64_t>(left - kUnitSteps, kLeastSteps));
        if (steps - at - n < kLeastSteps) n = steps - at;
        left -= n + kUnitSteps;
        return at + n;
    };
    // Blocks too short to be cut may leave much of every share: it grows until the CTAs are enough (5 x 9..43 tokens, 40/8 heads: 320 blocks
    // of a step on 296 CTAs, of which the last had 25, 274 us | 14.5)
    for (int64_t ctas = most_ctas + 1; o->force_kv_splits < 1 && ctas > most_ctas;) {
        int64_t left = share;
        ctas = 1;
        bool next = false;
        for (int i = 0; i < R && ctas <= most_ctas; ++i)
            for (int64_t r0 = 0; r0 < chunk_lens[i] && is_few(d, chunk_lens[i], walks); r0 += toks) {
                const int32_t steps = steps_for(prefix_lens[i] + std::min<int64_t>(r0 + toks, chunk_lens[i]));
                for (int64_t b = (int64_t)((G + heads - 1) / heads) * Hkv; b > 0; --b)
                    for (int32_t at = 0; at < steps; ctas += next) at = part_end(steps, at, left, next);
            }
        if (ctas > most_ctas) share += std::max<int64_t>(1, share / 16);
    }

    WppPlanHeader hd;
    std::memset(&hd, 0, sizeof(hd));
    size_t off = sizeof(WppPlanHeader);
    hd.off_q_offsets = (uint32_t)off;
    off += align_up(sizeof(int32_t) * (size_t)(R + 1), 16);
    hd.off_prefix = (uint32_t)off;
    off += align_up(sizeof(int32_t) * (size_t)(R + 1), 16);
    hd.off_units = (uint32_t)off;
    char* p = static_cast<char*>(plan_host);
    std::memset(p, 0, off);
    const int64_t unit_cap = ((int64_t)plan_host_bytes - (int64_t)off) / (int64_t)sizeof(WppUnit);
    WppUnit* us = reinterpret_cast<WppUnit*>(p + hd.off_units);
    std::vector<WppCombine> combines;
    int64_t n_units = 0, n_split = 0, key_steps = 0;
    std::vector<int32_t> first{0};           // of every CTA's units
    int64_t left = share;                    // of the current CTA's share
    int32_t slots = 0, slot0 = 0, slot_parts = 0, slot_row = 2 * WPP_HALF_M;      // the slots that have room: from slot0 on, row slot_row
    std::vector<int32_t> cuts;
    for (int i = 0; i < R; ++i) {
        const int64_t P = prefix_lens[i], C = chunk_lens[i];
        if (!is_few(d, C, walks)) continue;
        for (int64_t r0 = 0; r0 < C; r0 += toks) {
            const int32_t rows = (int32_t)std::min<int64_t>(toks, C - r0), steps = steps_for(P + r0 + rows);
            for (int32_t kvh = 0; kvh < Hkv; ++kvh) {
                for (int32_t h = 0; h < G; h += heads) {
                    const int32_t nh = std::min(heads, G - h);
                    cuts.assign(1, 0);
                    if (o->force_kv_splits >= 1) {
                        const int32_t n = std::min(o->force_kv_splits, steps);
                        for (int32_t q = 1; q <= n; ++q) cuts.push_back((int32_t)((int64_t)steps * q / n));
                    } else {
                        for (int32_t at = 0; at < steps;) {
                            bool next;
                            at = part_end(steps, at, left, next);
                            if (next) first.push_back((int32_t)(n_units + cuts.size() - 1));
                            cuts.push_back(at);
                        }
                    }
                    const int32_t parts = (int32_t)cuts.size() - 1;
                    if (n_units + parts > unit_cap) return WPP_ERR_PLAN_MISMATCH;
                    WppUnit u;
                    std::memset(&u, 0, sizeof(u));
                    u.request = i;
                    u.row0[0] = (int32_t)r0;
                    u.rows[0] = rows;
                    u.rows[1] = nh;
                    u.head[0] = kvh * G + h;
                    u.split_slot = -1;
                    u.pack = 1;
                    if (parts > 1) {
                        if (parts > slot_parts || slot_row + WPP_FEW_ROWS > 2 * WPP_HALF_M) {
                            slot0 = slots;
                            slot_parts = parts;
                            slot_row = 0;
                            slots += parts;
                        }
                        u.row0[1] = slot_row / WPP_HALF_M;
                        u.head[1] = slot_row % WPP_HALF_M;
                        slot_row += WPP_FEW_ROWS;
                        for (int32_t k = 0; k < nh; ++k)
                            combines.push_back({i, (int32_t)r0, rows, u.head[0] + k, slot0, parts, u.row0[1], u.head[1] + k * rows});
                    }
                    for (int32_t q = 0; q < parts; ++q) {
                        u.kv_begin = cuts[(size_t)q];
                        u.kv_end = cuts[(size_t)q + 1];
                        if (parts > 1) u.split_slot = slot0 + q;
                        u.cost = u.kv_end - u.kv_begin;
                        us[n_units++] = u;
                        key_steps += u.cost;
                        n_split += parts > 1;
                    }
                }
            }
        }
    }
    const int64_t n_few = n_units;

    // ---- tiles
    struct Tile { WppUnit u; int32_t steps; };
    std::vector<Tile> tiles;
    for (int i = 0; i < R; ++i) {
        const int64_t P = prefix_lens[i], C = chunk_lens[i];
        if (is_few(d, C, walks)) continue;
        const int32_t block = tile_rows(G);
        for (int64_t r0 = 0; r0 < C; r0 += block) {
            const int32_t rows = (int32_t)std::min<int64_t>(block, C - r0);
            Tile t;
            std::memset(&t, 0, sizeof(t));
            t.u.request = i;
            t.u.row0[0] = (int32_t)r0;
            t.steps = steps_for(P + r0 + rows);
            int32_t pack, per_tile;
            tile_heads(G, rows, &pack, &per_tile);
            if (rows <= WPP_HALF_M) {
                t.u.rows[0] = rows;
                t.u.rows[1] = per_tile == 2 * pack ? rows : 0;
                t.u.row0[1] = (int32_t)r0;
            } else {
                t.u.rows[0] = WPP_HALF_M;
                t.u.rows[1] = rows - WPP_HALF_M;
                t.u.row0[1] = (int32_t)r0 + WPP_HALF_M;
            }
            t.u.pack = pack;
            for (int32_t h = 0; h < Hq; h += per_tile) {
                t.u.head[0] = h;
                t.u.head[1] = h + (per_tile == 2 * pack ? pack : 0);
                tiles.push_back(t);
            }
        }
    }
    if ((int64_t)tiles.size() <= kTileOrderRounds * o->max_ctas)
        std::stable_sort(tiles.begin(), tiles.end(), [](const Tile& a, const Tile& b) { return a.steps > b.steps; });
    std::vector<std::pair<int64_t, int64_t>> counted;
    for (const Tile& t : tiles) counted.emplace_back(1, t.steps);
    const int64_t part_steps = tile_part_steps(counted, o->max_ctas, scratch_slots(d) - slots);
    for (Tile& t : tiles) {
        const int32_t parts = std::max(1, o->force_kv_splits >= 1 ? std::min(o->force_kv_splits, t.steps)
                                                                  : (int32_t)((t.steps + part_steps - 1) / part_steps));
        if (n_units + parts > unit_cap) return WPP_ERR_PLAN_MISMATCH;
        if (parts > 1)
            for (int hf = 0; hf < 2; ++hf)
                for (int32_t k = 0; k < std::min(t.u.pack, G) && t.u.rows[hf] > 0; ++k)
                    combines.push_back({t.u.request, t.u.row0[hf], t.u.rows[hf], t.u.head[hf] + k, slots, parts, hf, k * (WPP_HALF_M / t.u.pack)});
        for (int32_t q = 0; q < parts; ++q) {
            t.u.kv_begin = (int32_t)((int64_t)t.steps * q / parts);
            t.u.kv_end = (int32_t)((int64_t)t.steps * (q + 1) / parts);
            t.u.split_slot = parts > 1 ? slots + q : -1;
            t.u.cost = (t.u.kv_end - t.u.kv_begin) * ((t.u.rows[0] > 0) + (t.u.rows[1] > 0));
            us[n_units++] = t.u;
            key_steps += t.u.cost;
            n_split += parts > 1;
        }
        if (parts > 1) slots += parts;
    }
    if (n_units > 0x3fffffff) return WPP_ERR_INVALID_ARG;
    off += sizeof(WppUnit) * (size_t)n_units;
    if (o->force_kv_splits >= 1) {
        first.clear();
        for (int64_t u = 0; u < n_few; ++u) first.push_back((int32_t)u);
    }
    const int32_t few_ctas = n_few > 0 ? (int32_t)first.size() : 0;
    first.push_back((int32_t)n_few);
    if (off + align_up(sizeof(int32_t) * first.size(), 16) > plan_host_bytes) return WPP_ERR_PLAN_MISMATCH;
    hd.off_few_ctas = (uint32_t)off;
    std::memset(p + off, 0, align_up(sizeof(int32_t) * first.size(), 16));
    off += align_up(sizeof(int32_t) * first.size(), 16);
    hd.off_combine = (uint32_t)off;
    off += sizeof(WppCombine) * combines.size();
    hd.plan_bytes = align_up(off, 16);
    if (hd.plan_bytes > plan_host_bytes) return WPP_ERR_PLAN_MISMATCH;
    if (hd.plan_bytes > 0xffffffffu) return WPP_ERR_INVALID_ARG;       // (offsets are 32 bits)
    std::memcpy(p + hd.off_few_ctas, first.data(), sizeof(int32_t) * first.size());
    if (!combines.empty()) std::memcpy(p + hd.off_combine, combines.data(), sizeof(WppCombine) * combines.size());
    std::memset(p + off, 0, hd.plan_bytes - off);

    hd.magic = WPP_PLAN_MAGIC;
    hd.version = WPP_PLAN_VERSION;
    hd.desc_hash = wpp_desc_hash(d);
    hd.num_requests = R;
    hd.num_ctas = (int32_t)std::max<int64_t>(1, std::min<int64_t>(o->max_ctas, n_units - n_few));
    hd.num_units = (int32_t)n_units;
    hd.num_few_units = (int32_t)n_few;
    hd.num_few_ctas = few_ctas;
    hd.max_few_rows = max_rows;
    hd.num_combine = (int32_t)combines.size();
    hd.num_split_slots = slots;
    for (const WppCombine& c : combines) hd.max_combine_rows = std::max(hd.max_combine_rows, c.rows);
    hd.tile_m = o->tile_m;
    hd.tile_n = WPP_TILE_N;
    hd.head_dim = d->head_dim;
    hd.shape = 3;
    hd.total_new_tokens = T;
    hd.key_steps = key_steps;
    hd.flops = 4 * (int64_t)d->head_dim * Hq * pairs;
    hd.workspace_bytes = WPP_WS_HEADER_BYTES + align_up((size_t)slots * 2 * WPP_HALF_M * (d->head_dim + 1) * sizeof(float), 256);
    std::memcpy(p, &hd, sizeof(hd));
    int32_t* qo = reinterpret_cast<int32_t*>(p + hd.off_q_offsets);
    qo[0] = 0;
    for (int i = 0; i < R; ++i) qo[i + 1] = qo[i] + chunk_lens[i];
    int32_t* pp = reinterpret_cast<int32_t*>(p + hd.off_prefix);
    for (int i = 0; i < R; ++i) pp[i] = prefix_lens[i];

    info->num_tiles = n_units;
    info->num_split_tiles = n_split;
    info->num_combine_tiles = (int64_t)combines.size();
    info->num_ctas = std::max(few_ctas, n_units > n_few ? hd.num_ctas : 1);
    info->total_new_tokens = T;
    info->key_steps = key_steps;
    info->flops = hd.flops;
    info->shape = hd.shape;
    info->workspace_bytes = hd.workspace_bytes;
    info->plan_bytes = hd.plan_bytes;
    return WPP_OK;
}
