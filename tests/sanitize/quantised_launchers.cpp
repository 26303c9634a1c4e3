// Stand-ins for the launchers of the 4-bit cache in drivers that never call them: a call ends the run.
#include <cstdio>
#include <cstdlib>

#include "internal.h"

namespace sarathi {

static int unexpected(const char *what) {
    std::fprintf(stderr, "unexpected call of %s\n", what);
    std::exit(3);
}
int launch_kv_append_quantised(const sarathi_config &, const AppendMeta &, const void *, const void *, void *, int64_t, void *) {
    return unexpected("launch_kv_append_quantised");
}
int launch_kv_read_quantised(const sarathi_config &, const AppendMeta &, const void *, int64_t, void *, void *, void *) {
    return unexpected("launch_kv_read_quantised");
}
int launch_attention_quantised(const sarathi_config &, const AttnMeta &, const void *, const void *, int64_t, float, void *, int, void *) {
    return unexpected("launch_attention_quantised");
}

}  // namespace sarathi
