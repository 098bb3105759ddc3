// Plays launches of the register-tiled kernel whose workgroups share units, several at a time and started in many orders, and
// reports those that never end, and shares that leave out or repeat a chunk.  See test_shared_units.py.
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <random>
#include <vector>

#include "pconv_shares.h"

using namespace pconv;

struct Launch { int wgs, tiles, groups, n_chunks; bool one_set, by_ticket; };

constexpr int kXcds = 8;

// Units of the set that a workgroup belongs to, and how many workgroups that has.
static int set_units(const Launch &l, int set)
{
    const int tps = (l.tiles + 7) / 8;
    const int tiles = l.one_set ? l.tiles : std::max(0, std::min(l.tiles, (set + 1) * tps) - set * tps);
    return tiles * l.groups;
}
static int set_wgs(const Launch &l, int set) { return l.one_set ? l.wgs : (l.wgs - set + 7) / 8; }

// Every chunk of every unit once, a unit's pieces in order of the workgroups, each handed on by the one before.
static bool covers(const Launch &l)
{
    for (int set = 0; set < (l.one_set ? 1 : kXcds); ++set) {
        const int units = set_units(l, set);
        if (units == 0) continue;
        std::vector<int> at(units, 0), by(units, -1);
        for (int j = 0; j < set_wgs(l, set); ++j) {
            UnitShare s;
            if (!unit_share(j, set_wgs(l, set), units, l.n_chunks, s)) continue;
            const int n = unit_pieces(s, l.n_chunks);
            for (int p = 0; p < n; ++p) {
                const UnitPiece w = unit_piece(s, l.n_chunks, p);
                if (w.unit < 0 || w.unit >= units || w.c_begin != at[w.unit] || w.c_end <= w.c_begin || w.c_end > l.n_chunks) return false;
                if (w.c_begin > 0 && by[w.unit] != j - 1) return false;
                if (w.c_end < l.n_chunks && p != 0) return false;
                if (w.c_begin > 0 && p != n - 1) return false;
                at[w.unit] = w.c_end;
                by[w.unit] = j;
            }
        }
        for (int c : at) if (c != l.n_chunks) return false;
    }
    return true;
}

// Whether all launches end where XCD x has `places` workgroups at a time and takes the launches in the order order[x], each one's
// workgroups in order of their ids.  `turn`: which XCD starts its next workgroup.
static bool ends(const std::vector<Launch> &launches, int places, const std::vector<std::vector<int>> &order, std::mt19937 &turn)
{
    struct Running { int launch, xcd, j, piece, pieces, flag; UnitShare s; };
    std::vector<Running> running;
    std::vector<std::vector<int>> started(kXcds, std::vector<int>(launches.size(), 0));     // of each XCD's workgroups
    std::vector<std::vector<char>> handed(launches.size());
    std::vector<int> free_places(kXcds, places), tickets(launches.size(), 0);
    for (size_t k = 0; k < launches.size(); ++k) handed[k].assign(launches[k].wgs + 8, 0);
    long left = 0;
    for (const Launch &l : launches) left += l.wgs;
    for (bool moved = true; moved;) {
        moved = false;
        std::vector<int> xcds{0, 1, 2, 3, 4, 5, 6, 7};
        std::shuffle(xcds.begin(), xcds.end(), turn);
        for (int x : xcds) {
            if (free_places[x] == 0 || turn() % 4 == 0) continue;        // (a few of them at each step)
            for (int k : order[x]) {
                const Launch &l = launches[k];
                const int id = x + 8 * started[x][k];
                if (id >= l.wgs) continue;
                ++started[x][k];
                moved = true;
                const int set = l.one_set ? 0 : x, units = set_units(l, set);
                Running r{k, x, l.by_ticket ? tickets[k]++ : l.one_set ? id : id / 8, 0, 0, 0, {}};
                r.flag = l.one_set ? r.j : id;
                if (units == 0 || !unit_share(r.j, set_wgs(l, set), units, l.n_chunks, r.s)) { --left; break; }
                r.pieces = unit_pieces(r.s, l.n_chunks);
                --free_places[x];
                running.push_back(r);
                break;
            }
        }
        for (size_t i = 0; i < running.size();) {
            Running &r = running[i];
            const Launch &l = launches[r.launch];
            const UnitPiece w = unit_piece(r.s, l.n_chunks, r.piece);
            if (w.c_begin > 0 && !handed[r.launch][r.flag - (l.one_set ? 1 : 8)]) { ++i; continue; }
            moved = true;
            if (w.c_end < l.n_chunks) handed[r.launch][r.flag] = 1;
            if (++r.piece < r.pieces) { ++i; continue; }
            ++free_places[r.xcd];
            --left;
            r = running.back();
            running.pop_back();
        }
        if (!moved)                                      // (nobody was asked to start)
            for (int x = 0; x < kXcds; ++x)
                for (int k : order[x]) moved = moved || (free_places[x] > 0 && x + 8 * started[x][k] < launches[k].wgs);
    }
    return left == 0;
}

int main(int argc, char **argv)
{
    const bool by_id = argc > 1 && std::strcmp(argv[1], "by_id") == 0;       // the set of all workgroups with ids for tickets
    std::mt19937 rng(1909);
    long bad = 0, stuck = 0, played = 0;
    // 256 channels @56, one image: 13 tiles of 4 groups, 32 chunks; and others
    for (int wgs : {256, 250, 64, 9, 512})
        for (int tiles : {13, 1, 8, 49, 392})
            for (int n_chunks : {32, 5, 64}) {
                const int groups = tiles > 100 ? 1 : 4;
                if (int64_t(tiles) * groups * n_chunks / 2 < wgs) continue;
                for (bool one_set : {false, true}) {
                    const Launch l{wgs, tiles, groups, n_chunks, one_set, shares_by_ticket(one_set) && !by_id};
                    if (!covers(l)) { ++bad; std::printf("wgs=%d tiles=%d chunks=%d one_set=%d: chunks left out or repeated\n", wgs, tiles, n_chunks, one_set); }
                    for (int play = 0; play < 6; ++play) {
                        // two or three launches at once; XCDs agree about their order at first, then half do, then nobody
                        const std::vector<Launch> all(2 + play % 2, l);
                        std::vector<std::vector<int>> order(kXcds);
                        for (int x = 0; x < kXcds; ++x) {
                            for (size_t k = 0; k < all.size(); ++k) order[x].push_back(int(k));
                            if (play / 2 == 1 && x % 2) std::swap(order[x][0], order[x][1]);
                            if (play / 2 == 2) std::shuffle(order[x].begin(), order[x].end(), rng);
                        }
                        ++played;
                        if (!ends(all, (wgs + 7) / 8, order, rng)) {
                            ++stuck;
                            if (!by_id) std::printf("wgs=%d tiles=%d chunks=%d one_set=%d play=%d: never ends\n", wgs, tiles, n_chunks, one_set, play);
                        }
                    }
                }
            }
    std::printf("%ld played, %ld never end, %ld wrong shares\n", played, stuck, bad);
    return by_id ? (stuck == 0 || bad ? 1 : 0) : (stuck || bad ? 1 : 0);
}
