// Which rows a workgroup of attention has (attention.hpp), by looking at the texts' starts.  Plain C++ too: the search is tested on the CPU.
#pragma once
#include <stdint.h>

namespace pqt {
namespace {

constexpr int kLooks = 64;                 // starts that are looked at at once

// Rows begin .. begin + span of a text (of which `len` have tokens), and the first of those that a workgroup has.  Workgroup t of a head, of M rows each: text s
// has those from floor(start / M) + s on, which leaves every text one for each M rows it begins, without a table of them.
struct Rows {
    int64_t begin;
    int span, len, row0;
    bool mine;                             // false: nothing to do
    bool text;                             // false: rows of no text
    int64_t before;                        // rows before the first text that this workgroup clears, too
};

// `look` holds what its lanes see: look(lo, step) takes the starts of texts lo, lo + step .. (of text `texts` where there are no more: the rows behind the last one),
// each within 0 .. n, and with a step of 1 the texts' lengths; count(): how many lanes' texts are below `hi` and have workgroups up to t.
// Whatever order the places are in, the rows that it returns lie within the n there are; which ones is defined where they ascend.
template <int M, typename Look>
constexpr __attribute__((always_inline)) Rows rows_of_looks(Look& look, int64_t n, int texts, bool lengths, bool clear, int64_t t) {
    // the last text with floor(start / M) + s <= t: 64 of them looked at at once.  (s = texts: the rows behind the last one.)
    int lo = 0, hi = texts + 1;
    Rows r{};
    for (;;) {
        const int step = (hi - lo + kLooks - 1) / kLooks;
        look.look(lo, step);
        const int count = look.template count<M>(hi, t);
        if (count == 0) {                                      // rows before the first text
            // (a later look begins with a text that counts, unless the places do not ascend: these rows may lie past the last one then)
            r.begin = t * M < n ? t * M : n;
            r.span = n - r.begin < M ? (int)(n - r.begin) : M;
            r.mine = clear && r.span > 0;
            return r;
        }
        const int at = count - 1;
        lo += at * step;
        hi = hi < lo + step ? hi : lo + step;
        if (step > 1) continue;
        const int begin = look.start(at);
        int end = (int)n;
        r.text = lo < texts;
        if (r.text) end = at + 1 < kLooks ? look.start(at + 1) : look.start_of(lo + 1);
        if (end < begin) end = begin;
        r.begin = begin;
        r.span = end - begin;
        r.len = r.text ? r.span : 0;
        if (r.text && lengths) {
            const int tokens = look.tokens(at);
            if (tokens < r.len) r.len = tokens;
        }
        const int64_t row0 = (t - (begin / M + lo)) * M;
        r.before = lo == 0 && row0 == 0 && clear ? begin % M : 0;
        r.mine = r.before > 0 || (row0 >= 0 && row0 < r.span && (r.text || clear));    // (below 0: places that do not ascend)
        r.row0 = row0 < 0 ? 0 : (int)(row0 < r.span ? row0 : r.span);
        return r;
    }
}

}  // namespace
}  // namespace pqt
