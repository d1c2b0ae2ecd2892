// Argument checks and status messages shared by the library's C entry points.
#pragma once

#include <cmath>
#include <initializer_list>
#include <utility>

#include "mw.h"
#include "mw_kernels.h"

namespace mw {

constexpr int kMaxT = 1 << 24;  // keeps every in-kernel row * D index within 32 bits
constexpr float kLog2e = 1.4426950408889634f;

int fail(int code, const char* fmt, ...);
int ok();
bool aligned16(const void* p);
int check_ptrs(const char* fn, std::initializer_list<std::pair<const char*, const void*>> ptrs);
int hip_status(const char* fn, hipError_t e);
Strides contiguous(int H, int T, int D);
int check_view(const char* fn, const char* name, const mw_strides& s, int B, int H, int T, int D, bool output);
Strides to_internal(const mw_strides& s);
inline bool good_scale(float s) { return s > 0.f && std::isfinite(s); }

}  // namespace mw
