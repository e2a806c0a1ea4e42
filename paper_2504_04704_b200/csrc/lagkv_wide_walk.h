// How warps that meet at barriers inside a task go on from one task to the next.  Host and device code.
#pragma once

#ifdef __CUDACC__
#define LAGKV_WALK __host__ __device__ __forceinline__
#else
#define LAGKV_WALK inline
#endif

namespace lagkv {

// Every wait has a limit, and a wait may run out in one warp and not in the next one, so `ok` differs among warps that meet
// at barriers.  Inside a task a warp that has given up goes on without waiting and comes to every barrier; between tasks
// `agree` makes the outcome the same in all of them, the wait for the task itself included, so that they take the next task
// together or not at all.
//   told()    waits for the next task; false: the wait ran out
//   agree(ok) a barrier of these warps; true if `ok` is in all of them
template <class Told, class Agree>
LAGKV_WALK bool wide_go_on(bool& ok, Told&& told, Agree&& agree) {
    if (ok) ok = told();
    ok = agree(ok);
    return ok;
}

}  // namespace lagkv
