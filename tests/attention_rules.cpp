// The rules of lora_attention.h by which a call becomes launches, as functions that a test can call.  Built and loaded by test_attention_rules.py.
#include "lora_attention.h"

#include <cstdio>

// "few 16 cut", "wide 256 whole", "few 16 cut, wide 128 whole": the launches of a call
extern "C" const char *rule_forms(long long tokens, int group, int kv_heads, int requests, long long keys, long long most, int dim, int bits)
{
    static char text[100];
    const lora::AttendForms forms = lora::attend_forms(tokens, group, kv_heads, requests, keys, most, dim, bits == 8);
    int n = 0;
    for (int i = 0; i < forms.n; ++i)
        n += snprintf(text + n, sizeof text - n, "%s%s %d %s", i ? ", " : "", forms.f[i].columns <= 32 ? "few" : "wide", forms.f[i].columns, forms.f[i].cut ? "cut" : "whole");
    return text;
}

// shares of launch i, 0 where there is none
extern "C" int rule_shares(long long tokens, int group, int kv_heads, int requests, long long keys, long long most, int dim, int bits, int i)
{
    const lora::AttendForms forms = lora::attend_forms(tokens, group, kv_heads, requests, keys, most, dim, bits == 8);
    return i < forms.n ? forms.f[i].shares : 0;
}

// bytes that a call uses, and that it may use for any `most`
extern "C" long long rule_bytes(long long tokens, int group, int kv_heads, int requests, long long keys, long long most, int dim, int bits)
{
    const lora::AttendForms forms = lora::attend_forms(tokens, group, kv_heads, requests, keys, most, dim, bits == 8);
    size_t n = 0;
    for (int i = 0; i < forms.n; ++i) {
        const size_t b = lora::attend_parts_bytes(forms.f[i], kv_heads, dim);
        n = b > n ? b : n;
    }
    return (long long)n;
}
extern "C" long long rule_most_bytes(long long tokens, int group, int kv_heads, int requests, long long keys, int dim, int bits)
{
    return (long long)lora::attend_most_bytes(tokens, group, kv_heads, requests, keys, dim, bits == 8);
}
