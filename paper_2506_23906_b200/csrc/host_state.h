// Host-side state shared by the translation units of the library (defined in api.cu).
#pragma once
#include <atomic>

namespace mmv {

extern std::atomic<long long> g_launches;                 // kernels launched since the library was loaded
extern std::atomic<unsigned long long> g_budget_ns;       // time after which a device-side wait gives up

}  // namespace mmv
