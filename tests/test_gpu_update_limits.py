"""Updates of caches whose compactions need more shared memory than a launch has by default, from two host
threads at once: neither call takes away what the other one has asked for."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

from paper_2412_12094_b200 import api, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call,past", [("sepllm_cache_update_quant", (24000, 10300)),
                                       ("sepllm_cache_update", (24000, 20600))])
def test_two_threads_update_caches_of_different_sizes(call, past):
    """Every call is taken (a launch above the kernel's limit is refused by the runtime with an error)."""
    quant, d, w, s = call.endswith("quant"), 64, 8, 4
    sep = np.asarray(inputs.SEP_IDS, dtype=np.int32)
    jobs = []
    for n in past:
        desc = api.CacheDesc(1, 1, 1, d, 0, s, w, n + w)
        sizes = (api.sepllm_cache_bytes_quant if quant else api.sepllm_cache_bytes)(desc)
        state, Kc, Vc = (api.alloc_bytes(b) for b in (sizes[0], sizes[1], sizes[1]))
        api.sepllm_cache_init(desc, state)
        ids = torch.full((1,), 60, dtype=torch.int32, device="cuda")
        row = torch.ones((1, 1, d), dtype=torch.bfloat16, device="cuda")
        jobs.append((desc, state, Kc, Vc, ids, row, torch.cuda.Stream()))
    torch.cuda.synchronize()
    fn, start, codes, steps = getattr(api.lib(), call), threading.Barrier(2), [[], []], 3000

    def work(i):
        desc, state, Kc, Vc, ids, row, stream = jobs[i]
        p = [C.c_void_p(t.data_ptr()) for t in (state, Kc, Vc, ids, row)]
        args = (C.byref(desc), *p[:4], C.c_void_p(sep.ctypes.data), C.c_int32(sep.size), p[4], p[4],
                C.c_void_p(stream.cuda_stream))
        start.wait()
        for _ in range(steps):
            codes[i].append(fn(*args))
    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i, (_, state, *_) in enumerate(jobs):
        bad = sum(c != api.OK for c in codes[i])
        assert bad == 0, f"{bad} of {steps} updates of a cache with {past[i]} past entries were refused"
        assert api.read_cache_state(state)["next_pos"][0] == steps
