"""Calls of several host threads, each on a cache and a stream of its own."""
import threading

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise

pytestmark = pytest.mark.gpu


def test_extend_from_threads_with_unlike_numbers_of_slots():
    """The plan keeps two bitmaps over the slots in shared memory, more than a launch has by default; a thread with
    the smaller cache must not take it from one with the larger."""
    codes = {}

    def work(k, n_slots):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            cache = serve.PagedCache(1, 64, 1, 16, 64, n_slots, 2)
            slots, none = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
            granted, ws = torch.empty_like(slots), torch.empty(4096, dtype=torch.uint8, device="cuda")
        stream.synchronize()
        lib, seen = wise.load(), []
        for i in range(20000):
            seen.append(lib.wise_kv_extend(cache.ref, slots.data_ptr(), none.data_ptr(), 1, granted.data_ptr(),
                                           ws.data_ptr(), stream.cuda_stream))
            if i % 200 == 0:
                stream.synchronize()
        stream.synchronize()
        codes[k] = seen

    threads = [threading.Thread(target=work, args=(k, n)) for k, n in enumerate((1 << 18, 170000, 1 << 18, 180000))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(codes) == 4 and all(set(seen) == {wise.WISE_OK} for seen in codes.values())
    assert wise.wise_get_status() == wise.WISE_OK
