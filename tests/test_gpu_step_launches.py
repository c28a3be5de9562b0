"""RepairVerifyStep.launches_per_step against the kernels that a captured step holds."""
import ctypes as C

import pytest
import torch

from test_gpu_cache8 import DEV, Cache, _i32, cure  # noqa: F401

pytestmark = pytest.mark.gpu


def _kernels(graph):
    """Nodes of a captured graph."""
    n, lib = C.c_size_t(0), C.CDLL("libcuda.so.1")
    assert lib.cuGraphGetNodes(C.c_void_p(graph.raw_cuda_graph()), None, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("layers", [1, 3])
def test_launches(cure, layers):  # noqa: F811
    from paper_2608_00531_gb300.step import RepairVerifyStep, StepInputs
    B, K, V, R, Hq, Hkv = 2, 4, 256, 3, 4, 2
    n_max = 1 + K + R
    rnd = lambda *s: torch.randn(*s, device=DEV).bfloat16()  # noqa: E731
    cs = [Cache(cure, [40, 40], Hkv, 16, 3) for _ in range(layers)]
    step = RepairVerifyStep(B, K, V, 3, 1.0, R, 2, 1, layers, Hq, cs[0].kv, DEV, rope=cure.rope_desc(128, 1e4))
    codes = [[c.codes[w] for c in cs] for w in (0, 1)]
    scales = [[c.scales[w] for c in cs] for w in (0, 1)]
    wide = [[torch.zeros(c.codes[0].shape, dtype=torch.bfloat16, device=DEV) for c in cs] for _ in (0, 1)]
    logits = rnd(B, K, V), _i32([0] * B), _i32([20, 7]), None
    rows = [rnd(layers, B, n_max, h, 128) for h in (Hq, Hkv, Hkv)]
    given = StepInputs(*logits, *rows, rnd(B, n_max, V))
    projected = StepInputs(*logits, None, None, None, given.target_logits, rnd(layers, B, n_max, (Hq + 2 * Hkv) * 128))
    assert step.launches_per_step == 5 + layers
    counts = []
    for x in (given, projected):
        for caches, kw in ((wide, {}), (codes, dict(scales=scales))):
            step.run(x, *caches, **kw)
            graph = torch.cuda.CUDAGraph(keep_graph=True)
            with torch.cuda.graph(graph):
                step.run(x, *caches, **kw)
            assert step.launches_per_step == _kernels(graph)
            counts.append(step.launches_per_step)
    assert counts == [5 + layers, 8 + 2 * layers, 5 + 2 * layers, 8 + 3 * layers]
    host = StepInputs(*(t if t is None else t.cpu() for t in logits), *(t.cpu() for t in rows), given.target_logits.cpu())
    step.run_from_host(host, *wide)
    assert step.launches_per_step == 5 + layers and cure.cure_device_error() == 0
