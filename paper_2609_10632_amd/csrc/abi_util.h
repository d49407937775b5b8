// What the C ABI's sources share: error reporting and the workspace convention.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/numbat_conv.h"

namespace numbat {

// status with this thread's detail text
numbat_status fail(numbat_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
numbat_status ok();
numbat_status hip_fail(hipError_t e, const char* what);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Every non-empty workspace begins with a 256-byte header of counters for the kernels'
// grid-wide synchronisation (zero before a workspace's first use; every call leaves it
// zero); the op's own data follows.
constexpr size_t kWsHeader = 256;
inline size_t with_header(size_t body) { return body ? body + kWsHeader : 0; }
inline void* ws_body(void* ws) { return ws ? static_cast<char*>(ws) + kWsHeader : nullptr; }
numbat_status check_ws(void* ws, size_t have, size_t need);

constexpr int64_t kMaxIndex = (1ll << 31) - 1;

// numbat_workspace_size of the ops of numbat_mlp.h; false for another op
bool mlp_workspace_size(int op, const void* problem, size_t* bytes, numbat_status* st);
// and of numbat_attention.h
bool attention_workspace_size(int op, const void* problem, size_t* bytes, numbat_status* st);

}  // namespace numbat
