// The rules of lora_experts.h by which a call becomes launches, as functions that a test can call.  Built and loaded by test_experts_rules.py.
#include "lora_experts.h"

extern "C" long long rule_quantize_rows_at_once(int blocks) { return lora::quantize_rows_at_once(blocks); }
extern "C" int rule_quantize_blocks() { return lora::kQuantizeBlocks; }
