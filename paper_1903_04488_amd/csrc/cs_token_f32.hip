// Token log probabilities of logits in binary32.
#include "cs_token_kernels.h"

int cs::token_f32(TokenCall call, const TokenArgs& a) { return token<float>(call, a); }
