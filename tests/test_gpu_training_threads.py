"""Training operators called from several host threads at once, each on a stream of its own."""
import threading

import pytest
import torch

from tests.test_gpu_training_ops import fa, gen, randn

pytestmark = pytest.mark.gpu

BF16 = 1


def test_layer_norms_of_different_widths_from_several_threads():
    """One kernel with different amounts of shared memory: no call's launch goes by another call's size.  Calls of the
    C ABI, which runs without the interpreter's lock; 36 to 128 KB of parameters, four chunks a thread each."""
    f, rows, calls = fa(), 300, 10000
    wrong, go = [], threading.Barrier(4)

    def run(cols):
        x = randn(gen(cols), rows, cols, dtype=torch.bfloat16)
        w = randn(gen(cols + 1), cols, dtype=torch.bfloat16)
        want = f.fa_layer_norm_forward(x, w)[0]
        y = torch.empty_like(x)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        args = (x.data_ptr(), cols, None, 0, BF16, rows, cols, w.data_ptr(), None, BF16, 1e-5, y.data_ptr(), cols, None, 0, None, None,
                None, None, stream.cuda_stream)
        go.wait()
        for k in range(calls):
            code = f._lib.fa_layer_norm_forward(*args)
            if code != 0:
                wrong.append((cols, k, code))
            if k % 200 == 199:
                stream.synchronize()
        if not torch.equal(y, want):
            wrong.append((cols, "result"))

    threads = [threading.Thread(target=run, args=(cols,)) for cols in (4608, 4864, 8192, 16384)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, (len(wrong), wrong[:4])
