// What the host side of the dense operators launches for a size, from csrc/legend_internal.h, on the CPU.
#include "legend_internal.h"

extern "C" int64_t stub_adam_grid(int64_t units, int large) { return legend::adam_grid(units, large != 0); }
