/* include/sdp_layer.h from plain C: it compiles, links, refuses calls without
 * a context, and prints the descriptions' layouts. */
#include <stddef.h>
#include <stdio.h>

#include "sdp_layer.h"

int main(void) {
    sdp_rows r = {0};
    sdp_embed_desc em = {0};
    sdp_block_norm_desc bn = {0};
    sdp_block_norm_grads bg = {0};
    sdp_route_desc rt = {0};
    sdp_order_desc od = {0};
    sdp_expert_desc ex = {0};
    if (sdp_embed(NULL, &em, &r, &r, NULL) != SDP_ERR_INVALID_ARGUMENT) return 1;
    if (sdp_embed_backward(NULL, &em, &r, &r, 0, NULL) != SDP_ERR_INVALID_ARGUMENT) return 2;
    if (sdp_block_norm(NULL, &bn, &r, &r, &r, &r, NULL) != SDP_ERR_INVALID_ARGUMENT) return 3;
    if (sdp_block_norm_backward(NULL, &bn, &r, &r, &r, &r, &bg, NULL) != SDP_ERR_INVALID_ARGUMENT) return 4;
    if (sdp_route(NULL, &rt, NULL, NULL, NULL, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT) return 5;
    if (sdp_route_backward(NULL, &rt, NULL, NULL, NULL, NULL, 0, NULL) != SDP_ERR_INVALID_ARGUMENT) return 6;
    if (sdp_expert_order(NULL, &od, NULL, NULL, NULL, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT) return 7;
    if (sdp_expert_gather(NULL, &ex, &r, &r, NULL) != SDP_ERR_INVALID_ARGUMENT) return 8;
    if (sdp_expert_gather_backward(NULL, &ex, &r, &r, NULL) != SDP_ERR_INVALID_ARGUMENT) return 9;
    if (sdp_expert_combine(NULL, &ex, &r, NULL, &r, &r, NULL) != SDP_ERR_INVALID_ARGUMENT) return 10;
    if (sdp_expert_combine_backward(NULL, &ex, &r, NULL, &r, &r, NULL, NULL) != SDP_ERR_INVALID_ARGUMENT) return 11;
    if (sdp_last_error()[0] == 0) return 12;
    printf("sdp_rows %zu %zu\n", sizeof r, offsetof(sdp_rows, stride));
    printf("sdp_embed_desc %zu %zu %zu\n", sizeof em, offsetof(sdp_embed_desc, ids), offsetof(sdp_embed_desc, scale));
    printf("sdp_block_norm_desc %zu %zu %zu\n", sizeof bn, offsetof(sdp_block_norm_desc, scale),
           offsetof(sdp_block_norm_desc, pre_weight));
    printf("sdp_block_norm_grads %zu %zu %zu\n", sizeof bg, offsetof(sdp_block_norm_grads, dgate),
           offsetof(sdp_block_norm_grads, dpre_weight));
    printf("sdp_route_desc %zu %zu %zu\n", sizeof rt, offsetof(sdp_route_desc, scale),
           offsetof(sdp_route_desc, logit_stride));
    printf("sdp_order_desc %zu %zu\n", sizeof od, offsetof(sdp_order_desc, ends_type));
    printf("sdp_expert_desc %zu %zu\n", sizeof ex, offsetof(sdp_expert_desc, place));
    return 0;
}
