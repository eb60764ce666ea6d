#define OCTOPUS_D 256
#define OCTOPUS_AXES
#include "octopus_plans_append.inc"
