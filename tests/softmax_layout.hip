// What the passes of softmax cross-entropy write of each part of their scratch, beside what the layout gives it.  Host code: nothing is launched.
//
// stdin: lines "half forward N I O"; stdout: a line for each, "ok pieces piece last" or what is too small.
#include "../paper_1404_5997_amd/csrc/owt_softmax.hip"

// What the library's other files and the HIP runtime would give: linked without either, so that no device is asked for.
namespace owt {
owt_status fail(owt_status st, const char *, ...) { return st; }
int forced_tile() { return -1; }
int forced_split() { return 0; }
}  // namespace owt
extern "C" {
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
}

using namespace owt;

static const char *check(const SmLayout &l, int N, int I, int ol, bool forward, size_t &need, size_t &have)
{
    struct Part { const char *what; size_t at, bytes; };
    const size_t row = (size_t)l.isteps * (l.half ? 256 : 128), rows = forward ? N : (size_t)up(N, 64) * 64;
    size_t before = 0;
    for (int k = 0; k < l.pieces; k++) {
        const int cols = ol - k * l.piece < l.piece ? ol - k * l.piece : l.piece, psteps = up(cols, 64);
        const SmTileCost &z = kSmTiles[l.z.tile];
        // in the order in which the layout takes them: what lies behind a part is the next one that is not empty
        const size_t top = forward && l.z.splits <= 1 ? (size_t)up(cols, z.bn) * z.wn * N * sizeof(Top) : 0;
        size_t parts = partial_bytes(l.z, N, cols);
        if (!forward) {
            const size_t x = partial_bytes(l.dx, N, I), w = partial_bytes(l.dw, cols, I);
            parts = parts > x ? parts : x;
            parts = parts > w ? parts : w;
        }
        const Part all[] = {{"x", l.x, !forward || l.laid ? rows * row : 0},
                            {"w", l.w, l.laid ? cols * row : 0},
                            {"exponents of x", l.xexp, l.half ? (size_t)N * 4 : 0},
                            {"exponents of w", l.wexp, l.half ? (size_t)cols * 4 : 0},
                            {"least exponents of x", l.xlows, l.half && !forward ? (size_t)low_groups(rows) * 4 : 0},
                            {"least exponents of w", l.wlows, l.half && !forward ? (size_t)low_groups(cols) * 4 : 0},
                            {"least", l.least, l.half && !forward ? (size_t)8 : 0},
                            {"statistics", l.top, top ? before + top : 0},
                            {"labels' outputs", l.label_out, forward ? (size_t)N * 4 : 0},
                            {"dz", l.dz, !forward ? (size_t)N * psteps * 128 * l.planes : 0},
                            {"dz for dx", l.dz_dx, !forward && l.half ? (size_t)N * psteps * 256 : 0},
                            {"sums of dx", l.dxs, !forward && !l.half && l.pieces > 1 ? (size_t)N * I * 4 : 0},
                            {"sums of dbias", l.strips, !forward ? (size_t)strips_of(l.z, N) * cols * 4 : 0},
                            {"split sums", l.partial, parts}};
        before += top;
        constexpr int COUNT = sizeof(all) / sizeof(all[0]);
        for (int i = 0; i < COUNT; i++) {
            if (!all[i].bytes) continue;
            size_t end = l.total;
            for (int n = COUNT - 1; n > i; n--)
                if (all[n].bytes) end = all[n].at;
            need = all[i].bytes;
            have = end - all[i].at;
            if (all[i].at > end || need > have) return all[i].what;
        }
    }
    return nullptr;
}

int main()
{
    int half, forward, N, I, O;
    while (scanf("%d %d %d %d %d", &half, &forward, &N, &I, &O) == 5) {
        const owt_fc_desc d = {N, I, O, 1, 0, half ? OWT_F32 : OWT_BF16, 0};
        int ol;
        if (check_softmax(&d, ol) != OWT_OK) { printf("refused\n"); continue; }
        const SmLayout l(&d, ol, forward);
        if (l.few) { printf("few\n"); continue; }
        if (!l.fits()) { printf("refused\n"); continue; }
        size_t need = 0, have = 0;
        const char *what = check(l, N, I, ol, forward, need, have);
        if (what) printf("%s: %zu bytes of %zu, pieces of %d\n", what, need, have, l.piece);
        else printf("ok %d %d %d\n", l.pieces, l.piece, ol - (l.pieces - 1) * l.piece);
    }
    return 0;
}
