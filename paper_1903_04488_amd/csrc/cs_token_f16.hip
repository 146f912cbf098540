// Token log probabilities of logits in binary16.
#include "cs_token_kernels.h"

int cs::token_f16(TokenCall call, const TokenArgs& a) { return token<f16>(call, a); }
