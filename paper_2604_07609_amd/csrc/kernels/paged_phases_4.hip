// an engine's phases on a cache of 4 bits: norms, rotation and storage; attention
#include "../paged_phases.h"

PAGED_PHASES(64, 4)
PAGED_PHASES(128, 4)
