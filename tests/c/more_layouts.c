/* Prints the layouts of include/zq.h's structures of the optimizer's step and the policy
 * loss, and their codes, for comparison with a binding's.  Host only. */
#include <stddef.h>
#include <stdio.h>

#include "zq.h"

#define FIELD(type, field) \
  printf(#type "." #field " %zu %zu\n", offsetof(type, field), sizeof(((type*)0)->field))

int main(void) {
  printf("zq_adamw %zu\n", sizeof(zq_adamw));
  FIELD(zq_adamw, param);
  FIELD(zq_adamw, grad);
  FIELD(zq_adamw, grad_scales);
  FIELD(zq_adamw, m);
  FIELD(zq_adamw, m_scales);
  FIELD(zq_adamw, v);
  FIELD(zq_adamw, v_scales);
  FIELD(zq_adamw, out);
  FIELD(zq_adamw, out_scales);
  FIELD(zq_adamw, n);
  FIELD(zq_adamw, weight_decay);
  FIELD(zq_adamw, lr_scale);
  FIELD(zq_adamw, param_dtype);
  FIELD(zq_adamw, grad_dtype);
  FIELD(zq_adamw, state_dtype);
  FIELD(zq_adamw, out_dtype);
  FIELD(zq_adamw, grad_block);
  FIELD(zq_adamw, state_block);
  FIELD(zq_adamw, out_block);
  FIELD(zq_adamw, reserved);
  printf("zq_adamw_plan %zu\n", sizeof(zq_adamw_plan));
  FIELD(zq_adamw_plan, bytes);
  FIELD(zq_adamw_plan, pieces);
  FIELD(zq_adamw_plan, block_pieces);
  FIELD(zq_adamw_plan, count);
  FIELD(zq_adamw_plan, reserved);
  printf("zq_adamw_args %zu\n", sizeof(zq_adamw_args));
  FIELD(zq_adamw_args, lr);
  FIELD(zq_adamw_args, beta1);
  FIELD(zq_adamw_args, beta2);
  FIELD(zq_adamw_args, eps);
  FIELD(zq_adamw_args, step);
  FIELD(zq_adamw_args, max_norm);
  FIELD(zq_adamw_args, scale);
  printf("zq_policy %zu\n", sizeof(zq_policy));
  FIELD(zq_policy, old_logp);
  FIELD(zq_policy, advantages);
  FIELD(zq_policy, weights);
  FIELD(zq_policy, ref_logp);
  FIELD(zq_policy, clip_low);
  FIELD(zq_policy, clip_high);
  FIELD(zq_policy, kl);
  FIELD(zq_policy, scale);
  FIELD(zq_policy, grad_scale);
  FIELD(zq_policy, reserved);
  printf("ZQ_INT8 %d\nZQ_F8 %d\n", ZQ_INT8, ZQ_F8);
  return 0;
}
