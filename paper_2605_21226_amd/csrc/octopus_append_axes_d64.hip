#define OCTOPUS_D 64
#define OCTOPUS_AXES
#include "octopus_plans_append.inc"
