"""mpk_rows_*: what the entry points refuse, on graphs of the host alone (arguments are looked at before the graph is)."""
import pytest

import paper_2512_22219_amd as M
from tests.rows_util import RowsModel

P = 1 << 20   # an aligned address that nothing reads


@pytest.fixture(scope="module")
def model():
    return RowsModel(batch=3, host_only=True)


def _refused(call, *args, match):
    with pytest.raises(M.MpkError, match=match) as e:
        call(*args)
    assert e.value.status == M.MPK_ERR_INVALID_ARG


APPEND = dict(layer=0, n_seqs=1, n_rows=5, begin=P, slots=0, positions=P, qkv=P, kind=0, stride=512, q=P + 512, q_stride=256)
ATTEND = dict(layer=0, n_seqs=1, n_rows=5, begin=P, slots=0, positions=P, q=P, q_stride=256, out=P + 512, out_stride=256, work=P)
LOGITS = dict(n_rows=5, logits=P, kind=1, stride=64, tokens=P, n_top=4, logprobs=P, entropy=P, top_tokens=P, top_logprobs=P, work=P)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(n_rows=0), "host_only"), (dict(layer=2), "layer 2"), (dict(n_seqs=0), "n_seqs 0"),
    (dict(n_seqs=4), "n_seqs 4"), (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(begin=0), "NULL"), (dict(positions=0), "NULL"),
    (dict(qkv=0), "qkv"), (dict(qkv=P + 8), "qkv"), (dict(kind=2), "qkv_type"), (dict(stride=504), "qkv"), (dict(stride=516), "qkv"),
    (dict(q=0), "q_out"), (dict(q=P + 4), "q_out"), (dict(q_stride=248), "q_out"), (dict(q_stride=260), "q_out"),
    (dict(q=P), "in place"), (dict(q=P, q_stride=512, kind=1), "in place"), (dict(q=P, q_stride=512), "host_only")])
def test_append(model, change, match):
    _refused(model.graph.rows_append, *dict(APPEND, **change).values(), match=match)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(layer=2), "layer 2"), (dict(n_seqs=0), "n_seqs 0"), (dict(n_seqs=4), "n_seqs 4"),
    (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(begin=0), "NULL"), (dict(positions=0), "NULL"), (dict(q=0), "q is NULL"),
    (dict(q=P + 8), "q is NULL"), (dict(q_stride=248), "q: "), (dict(q_stride=257), "q: "), (dict(out=0), "out"),
    (dict(out=P + 520), "out"), (dict(out_stride=0), "out"), (dict(out=P), "out is q"), (dict(work=0), "workspace"),
    (dict(work=P + 4), "workspace")])
def test_attend(model, change, match):
    _refused(model.graph.rows_attend, *dict(ATTEND, **change).values(), match=match)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(logits=0), "logits"), (dict(logits=P + 2), "logits"),
    (dict(logits=P + 2, kind=0), "host_only"), (dict(logits=P + 1, kind=0), "logits"), (dict(kind=2), "logits_type"),
    (dict(stride=63), "stride"), (dict(tokens=0), "both"), (dict(logprobs=0), "both"), (dict(tokens=0, logprobs=0), "host_only"),
    (dict(n_top=33), "n_top"), (dict(top_tokens=0), "NULL"), (dict(top_logprobs=0), "NULL"),
    (dict(n_top=0, top_tokens=0, top_logprobs=0), "host_only"), (dict(work=0), "workspace"), (dict(work=P + 8), "workspace")])
def test_logprobs(model, change, match):
    _refused(model.graph.rows_logprobs, *dict(LOGITS, **change).values(), match=match)


@pytest.mark.parametrize("off", [1, 2])
@pytest.mark.parametrize("call,args,name,says", [
    ("rows_append", APPEND, "begin", "row_begin"), ("rows_append", APPEND, "slots", "slots"), ("rows_append", APPEND, "positions", "positions"),
    ("rows_attend", ATTEND, "begin", "row_begin"), ("rows_attend", ATTEND, "slots", "slots"), ("rows_attend", ATTEND, "positions", "positions"),
    ("rows_logprobs", LOGITS, "tokens", "tokens"), ("rows_logprobs", LOGITS, "logprobs", "logprobs"), ("rows_logprobs", LOGITS, "entropy", "entropy"),
    ("rows_logprobs", LOGITS, "top_tokens", "top_tokens"), ("rows_logprobs", LOGITS, "top_logprobs", "top_logprobs")])
def test_lists_and_results_off_their_elements(model, call, args, name, says, off):
    assert name in args
    _refused(getattr(model.graph, call), *dict(args, **{name: P + off}).values(), match=f"^.*{says} is not aligned")
    _refused(getattr(model.graph, call), *dict(args, **{name: P + 4}).values(), match="host_only")


def test_fewer_tokens_than_alternatives():
    g = RowsModel(vocab=8, host_only=True).graph
    _refused(g.rows_logprobs, *dict(LOGITS, n_top=9).values(), match="n_top 9")
    _refused(g.rows_logprobs, *dict(LOGITS, n_top=8).values(), match="host_only")


def test_no_rows_need_no_buffers():
    """An empty tensor has no address; what else the call says is still looked at."""
    g = RowsModel(host_only=True).graph
    append, attend, logits = dict(APPEND, n_rows=0, qkv=0, q_out=0), dict(ATTEND, n_rows=0, q=0, out=0), dict(LOGITS, n_rows=0, logits=0)
    for call, args in ((g.rows_append, append), (g.rows_attend, attend), (g.rows_logprobs, logits)):
        _refused(call, *args.values(), match="host_only")
    _refused(g.rows_append, *dict(append, n_seqs=0).values(), match="n_seqs")
    _refused(g.rows_attend, *dict(attend, layer=9).values(), match="layer")


def test_no_rows_need_no_buffers_none_of_them():
    """Every buffer of the rows is NULL, with strides of nothing; one name that a call does not have would be a mistake here."""
    g = RowsModel(host_only=True).graph
    for call, args, none in ((g.rows_append, APPEND, ("qkv", "stride", "q", "q_stride")), (g.rows_attend, ATTEND, ("q", "q_stride", "out", "out_stride", "work")),
                             (g.rows_logprobs, LOGITS, ("logits", "stride", "tokens", "logprobs", "entropy", "top_tokens", "top_logprobs", "work"))):
        empty = dict(args, n_rows=0, **dict.fromkeys(none, 0))
        assert list(empty) == list(args)
        _refused(call, *empty.values(), match="host_only")
        _refused(call, *dict(empty, n_rows=1).values(), match="NULL")


def test_a_cache_too_long_for_the_cuts():
    g = RowsModel(max_seq=(1 << 28) + 8, batch=1, host_only=True).graph
    for call in (lambda: g.rows_append(*APPEND.values()), lambda: g.rows_attend(*ATTEND.values())):
        with pytest.raises(M.MpkError, match="max_seq") as e:
            call()
        assert e.value.status == M.MPK_ERR_UNSUPPORTED
    _refused(g.rows_logprobs, *LOGITS.values(), match="host_only")


def test_a_serving_graph_and_a_task_dag():
    g = RowsModel(page=16, pages=99, serving=1, greedy_loop=1, host_only=True).graph
    _refused(g.rows_append, *APPEND.values(), match="server")
    _refused(g.rows_attend, *ATTEND.values(), match="server")
    _refused(g.rows_logprobs, *LOGITS.values(), match="server")
    dag = M.compile_dag(2, [(0, 1)])
    _refused(dag.rows_append, *APPEND.values(), match="DAG")
    _refused(dag.rows_attend, *ATTEND.values(), match="DAG")
    _refused(dag.rows_logprobs, *LOGITS.values(), match="DAG")


def test_constants():
    text = open(M.binding.__file__.replace("paper_2512_22219_amd/binding.py", "include/mpk.h")).read()
    assert "#define MPK_ROWS_WORKSPACE_BYTES (96u << 20)" in text and M.ROWS_WORKSPACE_BYTES == 96 << 20
    assert "#define MPK_ROWS_MAX_TOP 32u" in text and M.ROWS_MAX_TOP == 32
    assert "MPK_ROWS_BF16 = 0, MPK_ROWS_F32 = 1" in text and (M.ROWS_BF16, M.ROWS_F32) == (0, 1)
