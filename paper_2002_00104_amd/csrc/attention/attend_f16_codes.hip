#include "attend_launch.h"

namespace pwlq_attention {
template PWLQ_INTERNAL void attend_launch<f16, int8_t>(const Attend &, int, int, unsigned, hipStream_t);
}
