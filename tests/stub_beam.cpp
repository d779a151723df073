// The host side of beam search and of the cache in 4 bits on the runtime of stub_runtime.cpp: its calls in place of that file's.
#define calls tree_calls
#define main tree_main
#include "stub_runtime.cpp"
#undef calls
#undef main

static int calls(bool print) {
    int bad = 0;
    auto is = [&](const char* what, int rc) { if (rc) { ++bad; if (print) fprintf(stderr, "device %d: %s %d (%s)\n", device, what, rc, said.c_str()); } };
    int* i = (int*)64;
    char name[96];
    for (int dtype = 0; dtype < 3; ++dtype) {
        for (int V : {100, 32768, 131072})
            for (int B : {1, 20, 300}) {
                specdec_beam_select_args a = {(void*)4096, (float*)64, nullptr, nullptr, (float*)64, i, i, (void*)4096, 1ll << 40, V, dtype, B, 4, V, 8, 0};
                sprintf(name, "select %d %d x 4 x %d", dtype, B, V);
                is(name, specdec_beam_select(&a, nullptr));
            }
        for (int dim : {64, 128})
            for (int page : {16, 64})
                for (int T : {1, 2, 3, 4, 20, 60, 100, 300, 1024})
                    for (int B : {1, 40, 200})
                        for (int heads : {8, 32}) {
                            specdec_packed_cache c = {{(void*)4096, 3, 2, 8, dim, 1 << 12, page, 200, 8192 / page, 1ll << 32, 1ll << 31, 8 * page * dim / 2, dim / 2, page * dim / 2, i, i, i, i, i, i},
                                                      (void*)4096, 1ll << 32, 1ll << 31, 8 * page * dim / 16, page * dim / 16, nullptr};
                            specdec_tree_attention_args a = {(void*)4096, (void*)4096, heads * dim * T, heads * dim, dim, heads * dim * T, heads * dim, dim, B, T, heads, 0, i, (uint32_t*)64, 0, nullptr, 4000, 0.1f,
                                                             (void*)4096, 1ll << 40};
                            sprintf(name, "attention %d %d x %d, %d of %d wide, pages of %d", dtype, B, T, heads, dim, page);
                            is(name, specdec_packed_attention(&c, &a, dtype, nullptr));
                            if (T > 4 || heads > 8) continue;
                            specdec_packed_tokens t = {i, (void*)4096, (void*)4096, nullptr, 1 << 20, 8 * dim * T, 8 * dim, dim, B, 0, 2, dtype, T};
                            is("append", specdec_packed_cache_append(&c, &t, nullptr));
                            is("read", specdec_packed_cache_read(&c, &t, nullptr));
                            is("reorder", specdec_packed_cache_reorder(&c, i, i, B, 1, nullptr));
                            is("compact", specdec_packed_cache_compact(&c, i, B, i, 4, i, nullptr));
                        }
    }
    return bad;
}

int main() {
    const int first = calls(true), once = settings;
    device = 1;
    const int second = calls(true);
    printf("refused_on_the_first_device %d\nrefused_on_the_second_device %d\n", first, second);
    printf("settings_repeated %d\n", settings - 2 * once);
    const int before = settings;
    device = 0; calls(false);
    printf("settings_of_known_kernels %d\n", settings - before);
    device = 2; refuse_once = 1;                          // a device that refuses once is asked again
    const int refused = calls(false), again = calls(true);
    printf("not_refused_once %d\nrefused_after_a_failure %d\n", refused != 1, again);
    printf("wrong_launches %d\nno_launches %d\n", wrong, launches == 0);
}
