// The operators' choices of kernels (operator_kernels.h), for tests/test_operator_plans.py.
#include <vector>

#include "../paper_2211_13939_amd/csrc/operator_kernels.h"

using namespace tts;

extern "C" {
int plan_linear8(int rows, int in_dim, int out_dim, int two_bytes, int n_cu) { return (int)linear8_form(rows, out_dim, width8(in_dim) / E8_BLOCK, two_bytes, n_cu); }
// Of a launch of so many tiles: the sides of its grid, and how many tiles are not taken by one workgroup each.
int plan_linear8_grid(int tiles, int* across, int* down)
{
    const Linear8Grid g = linear8_grid(tiles);
    *across = g.across;
    *down = g.down;
    std::vector<unsigned char> taken(tiles);
    for (int y = 0; y < g.down; ++y)
        for (int x = 0; x < g.across; ++x) {
            const int t = linear8_tile(y * g.across + x, tiles);
            if (t < 0) return -1;
            if (t < tiles && taken[t] < 2) ++taken[t];
        }
    int wrong = 0;
    for (unsigned char n : taken) wrong += n != 1;
    return wrong;
}
int plan_cross_large(const int* q_len, const int* mem_len, int n, int group, int n_kv_heads, int n_cu)
{
    std::vector<CrossReq> r(n);
    for (int i = 0; i < n; ++i) r[i] = CrossReq{0, mem_len[i], 0, q_len[i], 0};
    return cross_many_large(r.data(), n, group, n_kv_heads, n_cu);
}
int plan_cross_many_rows() { return CROSS_MANY_ROWS; }
}
