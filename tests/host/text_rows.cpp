// Reads cases "M n clear with_lengths texts", starts (texts + 1 of them) and, where asked for, lengths from standard input, and prints for every workgroup
// "begin span len row0 mine text before": the lanes' looks at the starts, one lane after the other.
#include <cstdio>
#include <vector>

#include "../../paper_1702_05911_amd/csrc/text_rows.hpp"

struct Lanes {
    const std::vector<long long>&starts, &lengths;
    long long n;
    int texts, probe[pqt::kLooks], seen[pqt::kLooks], held[pqt::kLooks];

    int start_of(int s) const {
        const long long v = starts.at(s);
        return (int)(v < 0 ? 0 : v > n ? n : v);
    }
    void look(int lo, int step) {
        for (int lane = 0; lane < pqt::kLooks; ++lane) {
            probe[lane] = lo + lane * step;
            const int s = probe[lane] < texts ? probe[lane] : texts;
            seen[lane] = start_of(s);
            if (step == 1 && !lengths.empty()) {
                const long long v = lengths.at(s < texts ? s : texts - 1);
                held[lane] = (int)(v < 0 ? 0 : v > 0x7fffffff ? 0x7fffffff : v);
            }
        }
    }
    template <int M>
    int count(int hi, long long t) const {
        int c = 0;
        for (int lane = 0; lane < pqt::kLooks; ++lane) c += probe[lane] < hi && seen[lane] / M + probe[lane] <= t;
        return c;
    }
    int start(int lane) const { return seen[lane]; }
    int tokens(int lane) const { return held[lane]; }
};

template <int M>
void run(long long n, int clear, int texts, const std::vector<long long>& starts, const std::vector<long long>& lengths) {
    for (long long t = 0; t < n / M + texts + 1; ++t) {
        Lanes lanes{starts, lengths, n, texts, {}, {}, {}};
        const pqt::Rows r = pqt::rows_of_looks<M>(lanes, n, texts, !lengths.empty(), clear != 0, t);
        std::printf("%lld %d %d %d %d %d %lld\n", (long long)r.begin, r.span, r.len, r.row0, r.mine, r.text, (long long)r.before);
    }
}

int main() {
    int m, clear, with, texts;
    long long n;
    while (std::scanf("%d %lld %d %d %d", &m, &n, &clear, &with, &texts) == 5) {
        std::vector<long long> starts(texts + 1), lengths(with ? texts : 0);
        for (long long& v : starts)
            if (std::scanf("%lld", &v) != 1) return 1;
        for (long long& v : lengths)
            if (std::scanf("%lld", &v) != 1) return 1;
        if (m == 16) run<16>(n, clear, texts, starts, lengths);
        else if (m == 64) run<64>(n, clear, texts, starts, lengths);
        else run<128>(n, clear, texts, starts, lengths);
    }
    return 0;
}
