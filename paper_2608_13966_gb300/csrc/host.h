// Host-side state the translation units of the library share: the device's
// facts, a kernel's shared-memory limit and the failure-path hook.
#pragma once

#include <cstddef>
#include <cstdint>

#include "quasar.h"

namespace quasar {

// SM count of the current device and the address of its status word.
quasar_status host_device(int* n_sm, unsigned int** status);

// Let fn use up to the device's opt-in maximum of dynamic shared memory;
// UNSUPPORTED if `smem` is more than that.
quasar_status host_allow_smem(const void* fn, size_t smem);

// Clusters of `size` CTAs of fn the device holds at once (looked up once).
quasar_status host_max_clusters(const void* fn, int size, int threads, size_t smem, int* clusters);

// Bound on every device-side wait, and the quasar_debug_force_timeout value.
uint64_t host_timeout_ns();
uint64_t host_forced_timeout_ns();

}  // namespace quasar
