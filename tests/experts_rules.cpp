// The rules of lora_experts.h by which a call becomes launches, as functions that a test can call.  Built and loaded by test_experts_rules.py.
#include "lora_experts.h"

#include <cstdio>

extern "C" long long rule_quantize_rows_at_once(int blocks) { return lora::quantize_rows_at_once(blocks); }
extern "C" int rule_quantize_blocks() { return lora::kQuantizeBlocks; }

// "thin 2x4/4", "mid 4x2/1 once", "wide", "wide large": the kernel of a product by its tile, wavefronts or groups of them, and how it reads W
extern "C" const char *rule_product_form(int bits, int n_rows, int n_experts, int in, int out)
{
    static char text[64];
    const int pieces = bits == 16 ? in / 64 : (in + 127) / 128, met = lora::met_experts(n_experts, n_rows);
    const lora::ProductForm f = lora::product_form(bits == 8, n_rows, met, out, pieces);
    if (f.kind == lora::ProductForm::kWide)
        snprintf(text, sizeof text, lora::large_weights(met, out, pieces) ? "wide large" : "wide");
    else
        snprintf(text, sizeof text, "%s %dx%d/%d%s", f.kind == lora::ProductForm::kMid ? "mid" : "thin", f.rb, f.cb, f.groups, f.once ? " once" : "");
    return text;
}
