// The prompt kernel's index arithmetic (wq4_seen.h) on the CPU, item after item, against the definition of
// what a row sees.  Built with overflow checks that trap; a trap names the item.
//   prompt_walk <what> <items> <seed>     what: walk (lookups, list, masks), hidden (values that masks hide)
#include "wq4_seen.h"

#include <climits>
#include <csignal>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <unistd.h>
#include <vector>

using namespace wq4;

static char g_case[200];
static long g_bad;

static void trapped(int)
{
    if (write(2, g_case, strlen(g_case)) < 0 || write(2, ": a sum that an int does not hold\n", 34) < 0) _exit(3);
    _exit(2);
}

static void bad(const char* what, int at)
{
    if (++g_bad <= 10) fprintf(stderr, "%s: %s %d\n", g_case, what, at);
}

static bool sees(const View& a, long long pos, long long t)
{
    return t >= 0 && t < a.cap && t <= pos && (!a.window || t > pos - a.window || t < a.sinks);
}

static void walk(const View& a, const Seen& s, int pf, int ntok, int tok)
{
    std::vector<int> listed(a.cap, 0);
    for (int i = 0; i < s.tiles; ++i)
        for (int l = 0; l < kKeys; l += a.box) {              // a lookup a box
            const int t = s.token(i * kKeys + l);
            if (t > s.pl) continue;
            if (t < 0 || t + a.box > a.cap) {
                bad("page looked up for token", t);
                continue;
            }
            bool any = false;
            for (int d = 0; d < a.box; ++d) {
                ++listed[t + d];
                for (int r = 0; r < ntok && !any; ++r) any = sees(a, static_cast<long long>(pf) + r, t + d);
            }
            if (!any) bad("box read of which no row sees a token", t);
        }
    for (int t = 0; t < a.cap; ++t) {
        bool any = false;
        for (int r = 0; r < ntok && !any; ++r) any = sees(a, static_cast<long long>(pf) + r, t);
        if (any && listed[t] != 1) bad("token not listed once", t);
    }
    for (int i = 0; i < s.tiles; ++i)
        for (int base = 0; base < ntok; base += tok) {        // the row tiles of the item
            const int first = pf + base, last = first + std::min(tok, ntok - base) - 1;
            const bool all = sees_all(a, i, s.front, s.gap, first, last, s.pl);
            for (int r = base; r < std::min(base + tok, ntok); ++r) {
                const RowMask mask = row_mask(a, s, i, pf + r);
                for (int x = 0; x < kKeys; ++x) {
                    const bool got = all || (mask.word(x / 32) >> (x % 32) & 1u);
                    if (got != sees(a, static_cast<long long>(pf) + r, s.token(i * kKeys + x))) bad("mask of token", s.token(i * kKeys + x));
                }
            }
        }
}

// Which places of a tile the masked-value warp zeroes or looks at; false: it passes the tile by.
static bool places(const View& a, const Seen& s, int i, int last, std::vector<int>& zeroed, std::vector<int>& looked)
{
    if (sees_all(a, i, s.front, s.gap, s.pf, last, s.pl)) return false;
    auto mark = [i](std::vector<int>& v) {
        return [i, &v](int from, int to) {
            for (int r = std::min(std::max(from - i * kKeys, 0), kKeys); r < std::min(std::max(to - i * kKeys, 0), kKeys); ++r) v[r] = 1;
        };
    };
    hidden_places(a, s, last, mark(zeroed), mark(looked));
    return true;
}

static void hidden(const View& a, const Seen& s, int pf, int ntok)
{
    for (int i = 0; i < s.tiles; ++i) {
        std::vector<int> zeroed(kKeys, 0), looked(kKeys, 0);
        places(a, s, i, pf + ntok - 1, zeroed, looked);
        for (int x = 0; x < kKeys; ++x) {
            const int t = s.token(i * kKeys + x), seen_rows = [&] {
                int n = 0;
                for (int r = 0; r < ntok; ++r) n += sees(a, static_cast<long long>(pf) + r, t);
                return n;
            }();
            if (seen_rows && zeroed[x]) bad("zeroed, but seen: token", t);
            const bool copied = s.token(i * kKeys + x / a.box * a.box) <= s.pl;      // else the copy brings zeros
            if (copied && seen_rows < ntok && !zeroed[x] && !looked[x]) bad("not seen by every row, and passed by: token", t);
        }
    }
}

int main(int argc, char** argv)
{
    if (argc != 4) return 4;
    signal(SIGILL, trapped);
    signal(SIGTRAP, trapped);
    std::mt19937_64 g(strtoull(argv[3], nullptr, 10));
    auto in = [&](long long lo, long long hi) { return lo + static_cast<long long>(g() % static_cast<unsigned long long>(hi - lo + 1)); };
    for (int k = atoi(argv[2]); k > 0; --k) {
        View a;
        a.box = 16 << in(0, 3);
        a.cap = a.box * static_cast<int>(in(1, 1200 / a.box + 1));
        const long long windows[] = {0, in(1, 40), std::max(1ll, a.cap + in(-30, 30)), INT_MAX - in(0, 300), in(1, a.cap), in(1, a.cap)};
        const long long sinks[] = {0, in(0, 40), INT_MAX, in(0, a.cap)};
        const long long ends[] = {in(-50, 50), a.cap + in(-300, 300), INT_MAX - 1 - in(0, 500), (1ll << 30) + in(-500, 500), in(0, a.cap - 1),
                                  in(0, a.cap - 1)};
        const int tok = kKeys / static_cast<int>(in(1, 8)), ntok = in(0, 3) ? static_cast<int>(in(1, 2 * tok)) : 2 * tok;
        a.window = static_cast<int>(windows[in(0, 5)]);
        a.sinks = static_cast<int>(std::min<long long>(sinks[in(0, 3)], a.cap));
        const int pl = static_cast<int>(ends[in(0, 5)]), pf = pl - ntok + 1;
        snprintf(g_case, sizeof g_case, "rows at [%d, %d], cap %d, box %d, window %d, sinks %d", pf, pl, a.cap, a.box, a.window, a.sinks);
        const Seen s = seen_by(a, pf, pl);
        if (!strcmp(argv[1], "walk")) walk(a, s, pf, ntok, tok);
        else hidden(a, s, pf, ntok);
    }
    return g_bad != 0;
}
