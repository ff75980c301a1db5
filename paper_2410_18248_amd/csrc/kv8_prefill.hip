#include "internal.h"
namespace lamps {
hipError_t launch_kv8_prefill(const WindowArgs &, hipStream_t) { return hipErrorInvalidValue; }
}
