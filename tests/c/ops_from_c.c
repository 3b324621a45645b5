/* include/sdp_ops.h from plain C: it compiles, links, refuses a call without
 * a context, and prints the descriptions' layouts. */
#include <stddef.h>
#include <stdio.h>

#include "sdp_ops.h"

int main(void) {
    sdp_qk_norm_rope_desc qk = {0};
    sdp_grouped_desc gm = {0};
    sdp_distill_desc ds = {0};
    sdp_heads h = {0};
    if (sdp_qk_norm_rope(NULL, &qk, &h, &h, &h, &h, NULL) != SDP_ERR_INVALID_ARGUMENT) return 1;
    if (sdp_qk_norm_rope_backward(NULL, &qk, &h, &h, &h, &h, &h, &h, NULL, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT)
        return 2;
    if (sdp_grouped_matmul(NULL, &gm, NULL, NULL, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT) return 3;
    if (sdp_grouped_matmul_backward(NULL, &gm, NULL, NULL, NULL, NULL, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT) return 4;
    if (sdp_distill_loss(NULL, &ds, NULL, NULL, NULL, NULL, 0, NULL) != SDP_ERR_INVALID_ARGUMENT) return 5;
    if (sdp_distill_loss_backward(NULL, &ds, NULL, NULL, NULL, 0, NULL) != SDP_ERR_INVALID_ARGUMENT) return 6;
    if (sdp_last_error()[0] == 0) return 7;
    printf("sdp_heads %zu %zu\n", sizeof h, offsetof(sdp_heads, head_stride));
    printf("sdp_qk_norm_rope_desc %zu %zu %zu\n", sizeof qk, offsetof(sdp_qk_norm_rope_desc, eps),
           offsetof(sdp_qk_norm_rope_desc, k_weight));
    printf("sdp_grouped_desc %zu %zu %zu\n", sizeof gm, offsetof(sdp_grouped_desc, ends),
           offsetof(sdp_grouped_desc, dx_stride));
    printf("sdp_distill_desc %zu %zu %zu\n", sizeof ds, offsetof(sdp_distill_desc, teacher_logits),
           offsetof(sdp_distill_desc, label_weight));
    return 0;
}
