// What the source files behind petals_client.h and petals_finetune.h share of a client handle.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/petals_client.h"

// The handle's parameters and its workspace, nothing in which outlives a call: each call lays it out anew.
// It holds at least max_rows_per_call * (2 * hidden + 528) bytes.
struct ps_client_view {
    const petals_client_config *cfg;
    const petals_client_params *p;
    uint8_t *scratch;            // 256-byte aligned
    size_t scratch_bytes;
};
ps_client_view ps_view(const petals_client *client);
int ps_check_client_config(const petals_client_config *cfg);
