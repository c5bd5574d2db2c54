"""Calls on bf16 pages whose sequences have no rows at all (a captured call replayed while nobody has tokens), on the GPU: every
launch leaves the output, the queries and the pools as they are, and the next replay with rows is right."""
import numpy as np
import pytest
import torch

import rows_ref as rr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_rows import Case, D, _dev, _fill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


@pytest.mark.parametrize("a,g,B,max_new,rows,max_pos,window", [
    # single tokens and a few: a workgroup an item, equal parts, the list; then parts by count, by length, whole items
    (32, 8, 3, 1, 3, 200, 0), (4, 2, 1, 2, 2, 4000, 0), (32, 8, 12, 4, 40, 12000, 0), (32, 8, 12, 4, 40, 12000, 700),
    (16, 16, 12, 60, 88, 12000, 3000), (16, 16, 12, 60, 88, 12000, 0), (16, 1, 3, 64, 100, 40000, 0), (32, 8, 2, 20, 40, 1500, 300),
    (32, 8, 12, 9, 100, 100, 0)])
def test_calls_without_a_row(a, g, B, max_new, rows, max_pos, window):
    say(f"[no rows] a={a} g={g} B={B} max_new={max_new} rows={rows} max_pos={max_pos} window={window}")
    lens = [[90, 0, -1, 64, 1100, 63, 1, 65, 127, 128, 2, 500][i] % (max_pos - max_new) for i in range(B)]
    new = [min([17, 1, 2, 0, 9, 3, 1, 1, 5, 2, 7, 4][i], max_new) for i in range(B)]
    c = Case(a, g, lens, new, seed=90, rows=rows, stride=max_pos // 64 + 1)
    _fill(c)
    dev = c.cache.to_device()
    m = rr.model(a, g, dev, c.cache.n_pages, B, max(max_new, rows))
    if window:
        m.kvp_set_layer_window(0, window, 70)
    r, keep = rr.rows_of(lens, new, c.table, rows=rows, max_new=max_new, max_pos=max_pos)
    n = m.kvp_workspace_size(kb.KVP_PHASE_STEP, B, rows)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    x = _dev(c.x)
    q = _dev(c.x[:, :a].reshape(rows, -1))
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    p = x.data_ptr()

    def run():
        st = torch.cuda.current_stream().cuda_stream
        m.kvp_append(0, p, p + 2 * a * D, p + 2 * (a + g) * D, (a + 2 * g) * D, r, q_out.data_ptr(), st)
        m.kvp_attention(0, q.data_ptr(), r, out.data_ptr(), ws.data_ptr(), n, st)

    def call(f, cu):
        for t, u in zip(dev, c.cache.to_device()):
            t.copy_(u)
        keep["cu"].copy_(torch.tensor(np.asarray(cu), dtype=torch.int32))
        q_out.fill_(77.0)
        out.fill_(55.0)
        f()
        torch.cuda.synchronize()
        return q_out.clone(), out.clone(), c.cache.from_device(dev)

    real = call(run, c.cu)
    assert (real[0][: int(c.cu[-1])] != 77.0).any() and (real[1][: int(c.cu[-1])] != 55.0).any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for f in (run, graph.replay):
        for k in (0, rows // 2, rows):
            idle = call(f, [k] * (B + 1))
            assert (idle[0] == 77.0).all() and (idle[1] == 55.0).all() and idle[2].same(c.cache)
            again = call(f, c.cu)
            assert all(torch.equal(s.view(torch.int16), t.view(torch.int16)) for s, t in zip(again[:2], real[:2]))
            assert again[2].same(real[2])
