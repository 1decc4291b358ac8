"""Which kernels the sizes of the GPU tests of the experts' and adapters' edge
cases reach (csrc/expert_plans.hpp on the host, CPU only): every form."""
import test_expert_plans as plans
import test_gpu_expert_block_large as block
import test_gpu_expert_streams as streams
import test_gpu_lora_forms as lora


def _down(M, K, rank):
    if plans._call("down_rows", M, rank):
        return "rows"
    return 1 if rank <= 16 else 2 if rank <= 32 else 4, plans._call("down_slices", M, K, rank) > 1


def _up(M, N, K):
    return "skinny" if plans._call("up_skinny", M, N) else "tile"


def test_the_adapters_forms():
    reached = {(kind, _down(M, K, rank), _up(M, N, K)) for M, K, N, rank, kind in lora.FORMS}
    kinds = {"bf16", "fp16", "fp32"}
    assert {k for k, d, _ in reached if d == "rows"} == kinds
    assert {k for k, d, _ in reached if d != "rows"} == kinds
    assert {k for k, _, u in reached if u == "skinny"} == kinds
    assert {k for k, _, u in reached if u == "tile"} == kinds
    assert {d[0] for _, d, _ in reached if d != "rows"} == {1, 2, 4}  # 16-rank tiles per block
    assert {d[1] for _, d, _ in reached if d != "rows"} == {False, True}  # k in slices
    assert {(d == "rows", u) for _, d, u in reached} == {
        (True, "skinny"), (True, "tile"), (False, "skinny"), (False, "tile")}
    assert {plans._shape("lora_tile", M, N, K)[1] for M, K, N, *_ in lora.FORMS
            if _up(M, N, K) == "tile"} == {1, 2, 4}  # 32-row tiles per wave
    assert {M % 32 == 0 for M, *_ in lora.FORMS} == {False}
    assert any(K % 128 for _, K, *_ in lora.FORMS) and any(K % 128 == 0 for _, K, *_ in lora.FORMS)


def test_the_large_blocks_forms():
    """Every T of the block's tests takes the kernels of many rows; the largest
    one alphas staged in LDS."""
    for T in block.ROWS:
        pairs, E, width, hidden, rank = T * block.TOP_K, block.EXPERTS, 256, 512, 8
        assert pairs > 16384  # two launches for the order
        assert not plans._call("skinny", pairs, E, hidden)
        assert not plans._call("skinny", pairs, E, width)
        assert not plans._call("sum_by_rows", pairs, width, hidden)
        assert _down(T, width, rank) != "rows" and _up(T, width, width) == "tile"
    assert [plans._call("combine", T, block.EXPERTS, 256) > 0 for T in block.ROWS] == [False, True]


def test_the_streams_forms():
    M, K, N, _, rank = streams.LORA_MANY
    assert _down(M, K, rank) != "rows" and _up(M, N, K) == "tile"
    M, K, N, _, rank = streams.LORA_FEW
    assert _down(M, K, rank) == "rows" and _up(M, N, K) == "skinny"
    T, k, E, K, N = streams.SUM
    assert not plans._call("sum_by_rows", T * k, N, K)
    assert streams.GROUP[0] > 16384
