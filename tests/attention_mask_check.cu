// The mask's index arithmetic on the host: reads "batch q_len k_len causal window_left keys i j" lines and prints what query i and key j see
// of each other, as the kernels compute it (32-bit integers).
#include <cinttypes>
#include <cstdio>
#include "../paper_2609_02846_b200/csrc/attention.cuh"

int main() {
    long long q_len, k_len, window, keys, i, j;
    int causal;
    while (scanf("%lld %lld %d %lld %lld %lld %lld", &q_len, &k_len, &causal, &window, &keys, &i, &j) == 7) {
        ue5m3_attention_shape s{};
        s.batch = s.heads = s.kv_heads = 1;
        s.head_dim = 8;
        s.scale = 1.0f;
        s.q_len = q_len;
        s.k_len = k_len;
        s.causal = causal;
        s.window_left = window;
        const ue5m3::AttentionParams p = ue5m3::attention_params(s);
        printf("%d %d %d %d %d %d %d\n", p.key_lo((int)i), p.key_hi((int)i, (int)keys), p.query_lo((int)j), p.query_hi((int)j), p.first_key, p.first_query,
               p.queries_end((int)keys));
    }
    return 0;
}
