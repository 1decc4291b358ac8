"""The mixture-of-experts calls on streams of the caller's, at sizes that take
a workspace: calls issued on two streams at once from a third, with the
binding's own memory, give the bits of the same calls one after another."""
import numpy as np
import pytest
import torch

from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

GROUP = 200001, 300              # M, G
SUM = 1500, 2, 4, 1000, 700      # T, top_k, E, K, N
LORA_FEW = 64, 512, 600, 5, 8    # M, K, N, adapters, rank
LORA_MANY = 2100, 512, 600, 5, 8


def _words(g, *shape):
    return torch.from_numpy(g.integers(-2 ** 31, 2 ** 31, size=shape).astype(np.int32)).cuda()


def _group(seed):
    M, G = GROUP
    assert bnn.bnn_group_rows_workspace_size(M, G) > 0
    g = np.random.default_rng(seed)
    ids = torch.from_numpy(g.integers(-1, G, size=M).astype(np.int32)).cuda()
    return lambda **kw: bnn.bnn_group_rows(ids, G, **kw)


def _experts_sum(seed):
    T, k, E, K, N = SUM
    assert bnn.bnn_experts_sum_workspace_size(bnn.ExpertsDesc(T, k, E, N, K, 1)) > 0
    g = np.random.default_rng(seed)
    ids = torch.from_numpy(g.integers(0, E, size=(T, k)).astype(np.int32)).cuda()
    weights = torch.from_numpy(g.random((T, k)).astype(np.float32)).cuda()
    x, w = _words(g, T, bnn.words(K)), _words(g, E, N, bnn.words(K))
    offsets, order = bnn.bnn_group_rows(ids, E)
    return lambda **kw: (bnn.bnn_experts_sum(x, K, w, ids, weights, offsets, order, **kw),)


def _lora(sizes):
    def prepare(seed):
        M, K, N, L, rank = sizes
        assert bnn.bnn_bgemm_lora_workspace_size(bnn.LoraDesc(M, N, K, L, rank, 2, 2)) > 0
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        x, a, b = r(M, K), r(L, rank, K), r(L, N, rank)
        w = _words(np.random.default_rng(seed), N, bnn.words(K))
        ids = torch.randint(-1, L, (M,), generator=g, device="cuda").to(torch.int32)
        return lambda **kw: (bnn.bnn_bgemm_lora(x, w, ids, a, b, **kw),)
    return prepare


@pytest.mark.parametrize("prepare", [_group, _experts_sum, _lora(LORA_FEW), _lora(LORA_MANY)],
                         ids=["group", "experts_sum", "lora_few", "lora_many"])
def test_two_streams_at_once(prepare):
    calls = [prepare(seed) for seed in (1, 2)]
    want = [call() for call in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):  # both queues stay filled
        for i, (call, s) in enumerate(zip(calls, streams)):
            got[i].append(call(stream=s))
    torch.full((1 << 20,), -1, device="cuda")  # the current stream's allocations meanwhile
    torch.cuda.synchronize()
    for i in range(2):
        for result in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(result, want[i]))
