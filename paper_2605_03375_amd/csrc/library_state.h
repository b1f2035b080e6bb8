// What the library's host sources share: the error that tutti_last_hip_error returns, and the device's compute units.
#pragma once
namespace tutti {
__attribute__((visibility("hidden"))) int hip_failed(int hip_error);  // remembers it for this thread; returns TUTTI_EHIP
__attribute__((visibility("hidden"))) int compute_units();            // of the current device, or a negative TUTTI_E*
}  // namespace tutti
