/* Prints the layouts of include/zq.h's structures, and the codes that go in them, for
 * comparison with a binding's.  Host only. */
#include <stddef.h>
#include <stdio.h>

#include "zq.h"

#define FIELD(type, field) \
  printf(#type "." #field " %zu %zu\n", offsetof(type, field), sizeof(((type*)0)->field))

int main(void) {
  printf("zq_grad %zu\n", sizeof(zq_grad));
  FIELD(zq_grad, data);
  FIELD(zq_grad, scales);
  FIELD(zq_grad, out);
  FIELD(zq_grad, n);
  FIELD(zq_grad, dtype);
  FIELD(zq_grad, out_dtype);
  FIELD(zq_grad, block);
  FIELD(zq_grad, reserved);
  printf("zq_grad_plan %zu\n", sizeof(zq_grad_plan));
  FIELD(zq_grad_plan, bytes);
  FIELD(zq_grad_plan, norm_chunks);
  FIELD(zq_grad_plan, clip_chunks);
  FIELD(zq_grad_plan, count);
  FIELD(zq_grad_plan, reserved);
  printf("ZQ_F32 %d\nZQ_F16 %d\nZQ_BF16 %d\nZQ_I32 %d\nZQ_I64 %d\nZQ_INT4 %d\n", ZQ_F32, ZQ_F16, ZQ_BF16, ZQ_I32, ZQ_I64,
         ZQ_INT4);
  return 0;
}
