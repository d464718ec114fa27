"""Rules of the training operators' sources that no run shows reliably: reads in front of the wait for the kernel in front, waits that may
never end."""
import re

import pytest

from tests.test_kernel_sources import BARRIER, _body, _source


def _waits_first(body):
    """The kernel lets the one behind it start only past its own wait."""
    first = body.index("pdl_trigger();")
    return body.count("pdl_trigger();") == 1 and 0 <= body.find("pdl_wait();") < first


def test_tokens_are_pulled_to_l2_only_behind_the_sort():
    text = _source("dispatch.cu")
    assert _waits_first(_body(text, "sort_pairs_kernel"))
    body = _body(text, "spread_kernel")
    early = body[:body.index("pdl_wait();")]
    assert "prefetch_l2(" in early and "if (blockIdx.x < SPREAD_FIRST" in early and "i < a.ahead" in early
    assert not re.search(r"load_piece|a\.(perm|slots|weights|out|with)\b", early)     # nothing is read into registers, nothing written
    setters = [m.start() for m in re.finditer(r"a\.ahead = ", text)]
    call = _body(text, "emoe_dispatch")
    assert len(setters) == 1 and re.findall(r"launch_(\w+)\(", call)[-2:] == ["sort_pairs", "spread"] and "a.ahead = " in call


def test_kernels_behind_the_vectors_sum_wait_before_vectors_and_results():
    text = _source("lowrank_stream.cu")
    assert _waits_first(_body(text, "lowrank_sum_kernel"))
    up = _body(text, "lowrank_up_kernel")
    empty, roles = up[:up.index("list_rows<")], up[up.index("list_rows<"):]
    assert empty.index("pdl_wait();") < empty.index("pdl_trigger();") < empty.index("return;")
    assert not re.search(r"a\.(vec|out|base|scales|factor)\b", empty)
    assert roles.index("pdl_wait();") < roles.index("a.out +")
    assert roles.rindex("pdl_wait();") < roles.index("pdl_trigger();") < roles.index("load_vector<RP>(a.vec")
    stream = _body(text, "lowrank_stream_kernel")
    assert stream.index("if (!a.early) pdl_wait();") < stream.index("list_tiles<")
    assert stream.index("if (a.early) pdl_wait();") < stream.rindex("pdl_trigger();") < stream.index("a.vec +") < stream.index("a.planes +")
    for m in re.finditer(r"pdl_trigger\(\);", stream):                                 # every way out of the kernel has waited
        assert "pdl_wait();" in stream[:m.start()][-60:]
    many = _body(_source("lowrank.cu"), "launch_many")
    assert re.findall(r"launch_lowrank_(\w+)\(", many) == ["stream", "sum", "up", "stream"]
    assert many.index("launch_lowrank_up(") < many.index("x.early = 1;") and many.count("early") == 1


def test_the_join_reads_offsets_behind_kernels_that_waited():
    text = _source("lowrank.cu")
    join = _body(text, "lowrank_join_kernel")
    early = join[:join.index("pdl_wait();")]
    assert re.findall(r"a\.(\w+)", early) == ["off", "G", "n", "runs"]
    assert _waits_first(join) and _waits_first(_body(text, "lowrank_grad_kernel")) and _waits_first(_body(text, "lowrank_kernel"))
    back = _body(text, "emoe_lowrank_backward")
    assert [x for x in re.findall(r"launch_(\w+)", back)][-2:] == ["grads", "join"] and "launch_many" in back


@pytest.mark.parametrize("name", ["lowrank_stream.cu", "lowrank.cu", "lowrank.cuh"])
def test_no_barrier_among_warps_whose_waits_may_run_out(name):
    assert not re.search(BARRIER, _source(name))


@pytest.mark.parametrize("name", ["lowrank_stream.cu", "lowrank.cu", "dispatch.cu"])
def test_limits_of_shared_memory_go_through_the_shared_setter(name):
    assert "cudaFuncSetAttribute" not in _source(name)
