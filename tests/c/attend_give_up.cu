/* md_attend_cache with a limit for its waits, and a step that each warp takes for one whose copy did not land. */
#include "../../paper_2607_10582_gb300/csrc/md_attend.cu"

extern "C" __attribute__((visibility("default"))) md_status attend_give_up(const md_attend_cache_args *args, long long limit_ns,
                                                                           int lost_step) {
  return md::attend_cache(args, limit_ns, lost_step);
}
