// What the library's host sources share: the error that tutti_last_hip_error returns.
#pragma once
namespace tutti {
__attribute__((visibility("hidden"))) int hip_failed(int hip_error);  // remembers it for this thread; returns TUTTI_EHIP
}  // namespace tutti
