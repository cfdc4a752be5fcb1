// The count of kernel launches that pcr_launch_count returns; every source file of the library adds to it.
#pragma once
#include <stdint.h>

#include <atomic>

namespace pcr {
extern std::atomic<uint64_t> g_launches;
}
