// The operators' choices of kernels (operator_kernels.h), for tests/test_operator_plans.py.
#include "../paper_2211_13939_amd/csrc/operator_kernels.h"

using namespace tts;

extern "C" {
int plan_linear8(int rows, int in_dim, int out_dim, int two_bytes, int n_cu) { return (int)linear8_form(rows, out_dim, width8(in_dim) / E8_BLOCK, two_bytes, n_cu); }
}
