// kata_mixer.hip -- the operators around a recurrent mixer: short convolution, query-key
// norms with rotation, selective scan.  Host checks: kata_mixer_api.hpp.
#include "kata_conv.hpp"
#include "kata_qknorm.hpp"
#include "kata_ssm.hpp"
