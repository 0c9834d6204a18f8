"""The list of a prompt call's items (k_plan, for more than 128 sequences) on the CPU, its warps in
orders in which a write could overtake a read of shared memory."""
import ctypes

import pytest

import block_on_host as host

DRIVER = """
extern "C" void plan(int n, int T, int longest, int rows, int classes, const int* starts, int* count, PlanItem* items, int* err,
                     const int* order) {
  block::run(kPlanThreads, std::vector<int>(order, order + kPlanThreads / 32), 2 * (classes + 2) * sizeof(int),
             [=] { k_plan(n, T, longest, rows, classes, starts, Plan{count, items}, err); });
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    f = "kf_prompt_attention.cu"
    source = "constexpr int kPlanThreads = 1024;\n" + host.between(f, "struct PlanItem {", "// one sub-tile pair") + \
        host.between(f, "__global__ void __launch_bounds__(kPlanThreads) k_plan", "// ------------------------------------------------------------------ the products")
    return host.load(str(tmp_path_factory.mktemp("plan")), "plan", source, DRIVER)


@pytest.mark.parametrize("lens,rows", [([1] * 200, 128), ([5, 300, 0, 129] * 40, 128), ([700] * 3 + [1] * 1500, 256), ([0] * 140 + [1], 256)])
@pytest.mark.parametrize("order", range(3))
def test_every_item_is_listed(lib, lens, rows, order):
    starts = [0]
    for x in lens:
        starts.append(starts[-1] + x)
    n, T, longest = len(lens), starts[-1], max(lens)
    classes = max(1, -(-longest // rows))
    room = T // rows + n
    count, err, items = ctypes.c_int(-1), ctypes.c_int(0), (ctypes.c_int * (4 * room))(*[-1] * (4 * room))
    lib.plan(n, T, longest, rows, classes, (ctypes.c_int * (n + 1))(*starts), ctypes.byref(count), items, ctypes.byref(err), host.orders()[order])
    want = sorted((a, b - a, x) for a, b in zip(starts, starts[1:]) for x in range(-(-(b - a) // rows)))
    assert err.value == 0 and count.value == len(want)
    got = [tuple(items[4 * i: 4 * i + 3]) for i in range(count.value)]
    assert sorted(got) == want
    assert [x[2] for x in got] == sorted((x[2] for x in got), reverse=True)      # those of most key tiles first
