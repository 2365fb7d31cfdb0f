// What the C entries of the language-model operators check and report alike (operators.cu, layers.cu).
#pragma once
#include "../../include/tensair.h"
#include "operators.h"

namespace tensair {

constexpr uint64_t kMaxWidth = 1ull << 20, kMaxStride = (1ull << 31) - 1;

// Keeps `why` as what the calling thread's last refused or failed operator call said.
int refuse(int code, const char* why);
int launched(cudaError_t e);
#define TENSAIR_REQUIRE(cond, why) do { if (!(cond)) return refuse(TENSAIR_EINVAL, why); } while (0)

inline bool is_float_type(uint32_t type) { return type <= TENSAIR_FLOAT16; }
int check_rows(const tensair_rows* r, uint32_t d, bool empty, const char* null, const char* bad);
inline RowsView view_of(const tensair_rows& r) { return RowsView{r.data, (uint32_t)r.stride, r.type}; }
// Of the current device; 0: there is none.
int multiprocessors();

}  // namespace tensair
