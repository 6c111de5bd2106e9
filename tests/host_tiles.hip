// Device functions of the head's tiled products, compiled for the host and walked there lane by lane: which places of a result they write, which
// addresses they start from.  What a lane reads from LDS of other lanes is not modelled, so only places and addresses mean something.
#include <hip/hip_runtime.h>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#undef __device__
#define __device__ __attribute__((device)) __attribute__((host))
#define __builtin_amdgcn_wave_barrier() ((void)0)
#include "muon.hpp"

using namespace lc;
using namespace lc::head;

static constexpr bf16_t kUntouched = 0x7e00;   // a NaN in fp16: no value that is stored

// The most and the fewest waves that store a place of a symmetric n x n result's planes, by tiles of SIDE x SIDE and W waves.
template <int SIDE, int W, int PLANES>
static void walk_symmetric(int n, bool second) {
    constexpr int MT = SIDE / (16 * W), NT = SIDE / 64;
    const int ld = (int)round_up(n, 8), tiles = (n + SIDE - 1) / SIDE;
    const long long plane = (long long)n * ld;
    std::vector<bf16_t> out[2];
    std::vector<int> writers[2];
    for (int k = 0; k < 2; ++k) out[k].assign(PLANES * plane, kUntouched), writers[k].assign(PLANES * plane, 0);
    std::vector<char> lds(kEpiBytes<NT>);
    for (int tm = 0; tm < tiles; ++tm)
        for (int tn = 0; tn <= tm; ++tn)
            for (int wave = 0; wave < W; ++wave) {
                memset(lds.data(), 0x11, lds.size());
                PlaneEpi<PLANES, true> epi = {out[0].data(), second ? out[1].data() : nullptr, plane, PLANES * plane, ld, 1.f, 0.f, 0.f};
                epi.item(0);
                for (int lane = 0; lane < 64; ++lane) {
                    f32x16 acc[MT][NT];
                    for (auto &row : acc)
                        for (auto &v : row)
                            for (int e = 0; e < 16; ++e) v[e] = 1.f;
                    epi.run(acc, tm * SIDE + wave / 2 * MT * 32, tn * SIDE + wave % 2 * NT * 32, lane, n, n, 0, lds.data());
                }
                for (int k = 0; k < 2; ++k)
                    for (size_t i = 0; i < out[k].size(); ++i)
                        if (out[k][i] != kUntouched) ++writers[k][i], out[k][i] = kUntouched;
            }
    for (int k = 0; k < 1 + second; ++k) {
        int least = 1 << 30, most = 0;
        for (int w : writers[k]) least = std::min(least, w), most = std::max(most, w);
        printf("symmetric %d %d %d %d %d %d %d\n", SIDE, W, PLANES, n, k, least, most);
    }
}

// The same for tiles of 32 x 32: a workgroup's threads store four columns each, mirrored as well beside the diagonal.
template <int PLANES>
static void walk_blocks(int n) {
    const int ld = (int)round_up(n, 8), tiles = (n + 31) / 32;
    const long long plane = (long long)n * ld;
    std::vector<bf16_t> out(PLANES * plane, kUntouched);
    std::vector<int> writers(PLANES * plane, 0);
    const PlaneEpi<PLANES, true> epi = {out.data(), nullptr, plane, 0, ld, 1.f, 0.f, 0.f};
    for (int tm = 0; tm < tiles; ++tm)
        for (int tn = 0; tn <= tm; ++tn)
            for (int at = 0; at < 512; ++at) {
                const int r = at % 256 / 8, c = at % 8 * 4, a = at < 256 ? tm : tn, b = at < 256 ? tn : tm;
                if (at >= 256 && tm == tn) continue;
                float v[4] = {1.f, 1.f, 1.f, 1.f};
                epi.put4(a * 32 + r, b * 32 + c, v, n);
                for (size_t i = 0; i < out.size(); ++i)
                    if (out[i] != kUntouched) ++writers[i], out[i] = kUntouched;
            }
    printf("symmetric 32 4 %d %d 0 %d %d\n", PLANES, n, *std::min_element(writers.begin(), writers.end()), *std::max_element(writers.begin(), writers.end()));
}

// Where a wave's loads of a tile of N rows begin, in bytes from where they do in a contraction that begins at index 0, for one that begins at step kt;
// of both matrices, where a pair is read.  Every load moves by whole rows' bytes of kt steps.
template <int FORM, int N, int PL, int W>
static void walk_starts(int kt) {
    static bf16_t a[512 * 512], b[512 * 512];
    const bool pair = FORM == PAIR;
    Operand o = {a, pair ? b : a, 512, 0, 64, 0, 0};
    for (int wave = 0; wave < W; ++wave) {
        Stager<FORM, N, PL, W> first, later;
        first.init(o, 0, 0, 512, Format<PL>::B, wave, 5), later.init(o, 0, kt, 512, Format<PL>::B, wave, 5);
        const long long moved = later.base - first.base, moved2 = pair && W == 4 ? later.base2 - first.base2 : moved;
        const bool second = pair && W == 8 && wave >= 4;
        const bool inside = (const char *)later.base >= (const char *)(second ? b : a) && (const char *)later.base < (const char *)((second ? b : a) + 512 * 512);
        printf("start %d %d %d %d %lld %lld %lld %d\n", FORM, W, wave, kt, moved, moved2, (FORM == COL ? kt * kStep * o.ld : kt * kStep) * 2, inside);
    }
}

int main() {
    for (int kt : {0, 1, 3}) {
        walk_starts<ROW, 256, 1, 4>(kt), walk_starts<ROW, 256, 1, 8>(kt), walk_starts<PAIR, 256, 1, 4>(kt), walk_starts<PAIR, 128, 1, 4>(kt);
        walk_starts<PAIR, 256, BYTES, 8>(kt), walk_starts<COL, 256, 1, 4>(kt), walk_starts<COL, 256, 1, 8>(kt);
    }
    for (int n : {7, 32, 75}) walk_blocks<1>(n), walk_blocks<2>(n);
    for (int n : {64, 200, 256, 333, 520, 712}) {
        walk_symmetric<64, 4, 1>(n, false), walk_symmetric<64, 4, 2>(n, true);
        walk_symmetric<128, 4, 1>(n, true), walk_symmetric<128, 4, 2>(n, false);
        walk_symmetric<192, 4, 1>(n, false), walk_symmetric<192, 4, 2>(n, true);
        walk_symmetric<256, 8, 1>(n, true), walk_symmetric<256, 8, 2>(n, true);
    }
    return 0;
}
