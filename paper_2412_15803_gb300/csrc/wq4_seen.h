// wq4_seen.h -- which tokens the rows of a prompt see, as prompt_attn_kernel walks them:
// the list of key tiles, the masks of a row in a tile, and the places of a tile whose
// values a mask hides.  Plain index arithmetic, compiled as C++ too, so that a test can
// run it on the CPU.
//
// Positions and lengths come from device memory and may be anything up to 2^31 - 1:
// no sum here passes an int, whatever they are (cap is below 2^30, a tile 128).
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define WQ4_SEEN __device__ __forceinline__
#else
#include <algorithm>
#define WQ4_SEEN inline
#endif

namespace wq4 {

#ifndef __CUDACC__
using std::max;
using std::min;
#endif

constexpr int kKeys = 128;           // keys of a tile

// What the rows of one call see: the row at position i the tokens t <= i, t < cap with
// window == 0 or t > i - window or t < sinks.
struct View {
    int cap;                         // tokens of a sequence that the page table has room for, a multiple of box
    int box;                         // cache rows of one copy: a page's, or the part of it that divides a tile
    int window, sinks;               // window 0: none; sinks <= cap
};

// The first token that the window shows a row at `pos` (window >= 1).
WQ4_SEEN int window_first(const View& a, int pos) { return pos < a.window ? 0 : pos - a.window + 1; }

// What the rows at positions [pf, pl] of one item see: a list of tokens in tiles
// of 128.  Place x of the list is token x, from `front` on token x + gap: the
// boxes (box tokens) between the sinks and the window are not in the list, so
// that a few sinks share a tile with the window's first tokens.
struct Seen {
    int pf, pl, tiles, front, gap;
    WQ4_SEEN int token(int x) const { return x + (x >= front ? gap : 0); }
};

WQ4_SEEN Seen seen_by(const View& a, int pf, int pl)
{
    Seen s;
    s.pf = pf;
    s.pl = min(pl, a.cap - 1);
    const int all = max(s.pl + 1, 0);
    s.front = s.gap = 0;
    if (a.window) {
        // (a window that begins behind the table's end shows nothing: it might as well begin there)
        const int front = (min(a.sinks, all) + a.box - 1) & -a.box, first = min(window_first(a, pf), a.cap) & -a.box;
        if (first > front) {
            s.front = front;
            s.gap = first - front;
        }
    }
    // (positions beyond the table's end may leave the sinks alone); an item without keys still writes its zeros
    s.tiles = max(1, (max(all - s.gap, min(s.front, all)) + kKeys - 1) / kKeys);
    return s;
}

// Whether the rows at [pf, pl] see every key of tile i of the list; end: the last token of the cache.
WQ4_SEEN bool sees_all(const View& a, int i, int front, int gap, int pf, int pl, int end)
{
    const int x = i * kKeys, t = x + (x >= front ? gap : 0);
    return t + kKeys - 1 <= min(pf, end) && (!a.window || t >= window_first(a, pl) || t + kKeys <= a.sinks) &&
           (x >= front || x + kKeys <= front);
}

// The lowest n bits (none for n <= 0, all for n >= 32).
WQ4_SEEN uint32_t first_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : (1u << max(n, 0)) - 1u; }

// What the row at `pos` sees of tile i of the list, a bit a key: those up to hi, less
// those from sk to lo; before fr the sinks that lie in front.
struct RowMask {
    int hi, lo, sk, fr, fs;
    WQ4_SEEN uint32_t word(int c) const          // keys [32 c, 32 c + 32)
    {
        return first_bits(fs - 32 * c) |
               (first_bits(hi - 32 * c) & ~first_bits(fr - 32 * c) & (~first_bits(lo - 32 * c) | first_bits(sk - 32 * c)));
    }
};

WQ4_SEEN RowMask row_mask(const View& a, const Seen& s, int i, int pos)
{
    const int t0 = i * kKeys + s.gap;
    return {min(pos, s.pl) - t0 + 1, a.window ? window_first(a, pos) - t0 : 0, a.window ? a.sinks - t0 : 0, s.front - i * kKeys,
            min(min(a.sinks, pos + 1), s.front) - i * kKeys};
}

// The places [from, to) of the list whose values a mask hides: zero(from, to) of those
// that no row of the item sees but a copy brings, look(from, to) of those that some see.
// last: the position of the item's last row (s.pl, but where that lies behind the table's end).
template <typename Zero, typename Look>
WQ4_SEEN void hidden_places(const View& a, const Seen& s, int last, Zero zero, Look look)
{
    const int pf = s.pf, pl = s.pl, gap = s.gap;
    // Seen by no row: behind pl in its box, and between the sinks and the window in
    // theirs.  Seen by some: behind pf, and up to the window's beginning at the last row.
    zero(pl + 1 - gap, (pl / a.box + 1) * a.box - gap);
    look(max(pf, -1) + 1 - gap, pl + 1 - gap);
    if (a.window) {
        const int gone = window_first(a, pf);
        if (gap) {
            zero(a.sinks, s.front);
            zero(s.front, gone - gap);
        } else {
            zero(a.sinks, gone);
        }
        look(max(a.sinks, gone) - gap, min(window_first(a, last), pf + 1) - gap);
    }
}

}  // namespace wq4
