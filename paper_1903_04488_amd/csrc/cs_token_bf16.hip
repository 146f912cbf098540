// Token log probabilities of logits in bf16.
#include "cs_token_kernels.h"

int cs::token_bf16(TokenCall call, const TokenArgs& a) { return token<bf16>(call, a); }
