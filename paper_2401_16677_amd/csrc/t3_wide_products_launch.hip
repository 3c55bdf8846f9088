// Launches of the wide-tile kernel on operands in 8 bits and by group (see t3_wide_launch.hip).
#include "t3_wide_launch.hip"
