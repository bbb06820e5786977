// an engine's phases on a cache of 16 bits: norms, rotation and storage; attention
#include "../paged_phases.h"

PAGED_PHASES(64, 16)
PAGED_PHASES(128, 16)
