#define OCTOPUS_D 128
#define OCTOPUS_AXES
#include "octopus_plans_append.inc"
