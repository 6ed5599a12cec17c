"""mpk_tree_*: what the entry points refuse, on graphs of the host alone (arguments are looked at before the graph is)."""
import pytest

import paper_2512_22219_amd as M
from tests.rows_util import RowsModel

P = 1 << 20   # an aligned address that nothing reads
R = [P + 4096 * (i + 1) for i in range(4)]   # ... and others


@pytest.fixture(scope="module")
def model():
    return RowsModel(batch=3, host_only=True)


def _refused(call, *args, match, status=M.MPK_ERR_INVALID_ARG):
    with pytest.raises(M.MpkError, match=match) as e:
        call(*args)
    assert e.value.status == status


APPEND = dict(layer=0, n_seqs=1, n_rows=5, begin=P, slots=0, positions=P, parents=P, qkv=P, kind=0, stride=512, q=P + 512, q_stride=256)
ATTEND = dict(layer=0, n_seqs=1, n_rows=5, begin=P, slots=0, positions=P, parents=P, q=P, q_stride=256, out=P + 512, out_stride=256, work=P)
VERIFY = dict(n_seqs=1, n_rows=5, begin=P, parents=P, tokens=P, logits=P, kind=1, stride=64, draft=P, draft_stride=64, flags=0,
              temperatures=P, uniforms=P, lengths=R[0], path=R[1], next=R[2], logprobs=R[3], work=P)
KEEP = dict(n_seqs=1, n_rows=5, begin=R[0], slots=0, positions=P, lengths=R[1], path=R[2], out=P + 512)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(n_rows=0, parents=0), "host_only"), (dict(parents=0), "NULL"), (dict(parents=P + 2), "parents"), (dict(layer=2), "layer 2"),
    (dict(n_seqs=0), "n_seqs 0"), (dict(n_seqs=4), "n_seqs 4"), (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(begin=0), "NULL"),
    (dict(positions=0), "NULL"), (dict(qkv=0), "qkv"), (dict(kind=2), "qkv_type"), (dict(stride=504), "qkv"), (dict(q_stride=260), "q_out"),
    (dict(q=P), "in place"), (dict(q=P, q_stride=512), "host_only")])
def test_append(model, change, match):
    _refused(model.graph.tree_append, *dict(APPEND, **change).values(), match=match)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(n_rows=0, parents=0), "host_only"), (dict(parents=0), "NULL"), (dict(parents=P + 1), "parents"), (dict(layer=2), "layer 2"),
    (dict(n_seqs=4), "n_seqs 4"), (dict(positions=0), "NULL"), (dict(q=P + 8), "q is NULL"), (dict(q_stride=248), "q: "), (dict(out=0), "out"),
    (dict(out_stride=0), "out"), (dict(out=P), "out is q"), (dict(work=0), "workspace"), (dict(work=P + 4), "workspace")])
def test_attend(model, change, match):
    _refused(model.graph.tree_attend, *dict(ATTEND, **change).values(), match=match)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(n_rows=0), "host_only"), (dict(n_seqs=0), "n_seqs 0"), (dict(n_seqs=4), "n_seqs 4"),
    (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(begin=0), "NULL"), (dict(parents=0), "NULL"), (dict(tokens=0), "NULL"),
    (dict(lengths=0), "NULL"), (dict(path=0), "NULL"), (dict(next=0), "NULL"), (dict(logprobs=0), "host_only"), (dict(logits=0), "logits"),
    (dict(logits=P + 2), "logits"), (dict(logits=P + 2, kind=0), "host_only"), (dict(logits=P + 1, kind=0), "logits"),
    (dict(kind=2), "logits_type"), (dict(stride=63), "row stride"), (dict(draft_stride=63), "draft_probs"), (dict(draft=P + 2), "draft_probs"),
    (dict(draft=0, draft_stride=0), "host_only"), (dict(flags=2), "flags"), (dict(flags=1), "host_only"),
    (dict(flags=1, draft=0), "MPK_TREE_DRAWN_ONCE"), (dict(uniforms=0), "NULL"), (dict(temperatures=0, uniforms=0), "host_only"),
    (dict(work=0), "workspace"), (dict(work=P + 8), "workspace")])
def test_verify(model, change, match):
    _refused(model.graph.tree_verify, *dict(VERIFY, **change).values(), match=match)


@pytest.mark.parametrize("change,match", [
    ({}, "host_only"), (dict(out=0), "host_only"), (dict(out=P), "positions_out is positions"), (dict(n_seqs=0), "n_seqs 0"),
    (dict(n_seqs=4), "n_seqs 4"), (dict(n_rows=(1 << 24) + 1), "n_rows"), (dict(begin=0), "NULL"), (dict(positions=0), "NULL"),
    (dict(lengths=0), "NULL"), (dict(path=0), "NULL"), (dict(n_rows=0, lengths=0, path=0), "host_only")])
def test_keep(model, change, match):
    _refused(model.graph.tree_keep, *dict(KEEP, **change).values(), match=match)


@pytest.mark.parametrize("off", [1, 2])
@pytest.mark.parametrize("call,args,name,says", [
    ("tree_append", APPEND, "begin", "row_begin"), ("tree_append", APPEND, "slots", "slots"), ("tree_append", APPEND, "positions", "positions"),
    ("tree_append", APPEND, "parents", "parents"), ("tree_attend", ATTEND, "parents", "parents"), ("tree_attend", ATTEND, "begin", "row_begin"),
    ("tree_verify", VERIFY, "begin", "row_begin"), ("tree_verify", VERIFY, "parents", "parents"), ("tree_verify", VERIFY, "tokens", "tokens"),
    ("tree_verify", VERIFY, "draft", "draft_probs"), ("tree_verify", VERIFY, "temperatures", "temperatures"),
    ("tree_verify", VERIFY, "uniforms", "uniforms"), ("tree_verify", VERIFY, "lengths", "lengths"), ("tree_verify", VERIFY, "path", "path"),
    ("tree_verify", VERIFY, "next", "next_tokens"), ("tree_verify", VERIFY, "logprobs", "logprobs"), ("tree_keep", KEEP, "begin", "row_begin"),
    ("tree_keep", KEEP, "slots", "slots"), ("tree_keep", KEEP, "positions", "positions"), ("tree_keep", KEEP, "lengths", "lengths"),
    ("tree_keep", KEEP, "path", "path"), ("tree_keep", KEEP, "out", "positions_out")])
def test_lists_and_results_off_their_elements(model, call, args, name, says, off):
    assert name in args
    _refused(getattr(model.graph, call), *dict(args, **{name: P + 16 + off}).values(), match=f"^.*{says} is not aligned")
    _refused(getattr(model.graph, call), *dict(args, **{name: P + 20}).values(), match="host_only")


@pytest.mark.parametrize("result,on,match", [
    ("lengths", "begin", "lengths is row_begin"), ("path", "parents", "path is parents"), ("path", "tokens", "path is tokens"),
    ("next", "temperatures", "next_tokens is temperatures"), ("logprobs", "uniforms", "logprobs is uniforms"), ("logprobs", "logits", "logprobs is logits"),
    ("logprobs", "draft", "logprobs is draft_probs"), ("path", "lengths", "path is lengths"), ("next", "path", "next_tokens is path"),
    ("logprobs", "next", "logprobs is next_tokens")])
def test_results_on_what_is_read(model, result, on, match):
    apart = dict(VERIFY, **{n: P + 4096 * (i + 9) for i, n in enumerate(VERIFY) if VERIFY[n] == P})
    _refused(model.graph.tree_verify, *apart.values(), match="host_only")
    _refused(model.graph.tree_verify, *dict(apart, **{result: apart[on]}).values(), match=match)


@pytest.mark.parametrize("on,name", [("begin", "row_begin"), ("slots", "slots"), ("positions", "positions"), ("lengths", "lengths"), ("path", "path")])
def test_new_positions_on_what_is_read(model, on, name):
    _refused(model.graph.tree_keep, *dict(KEEP, **{on: P + 512}).values(), match=f"positions_out is {name}")


def test_a_vocabulary_too_large():
    g = RowsModel(vocab=(1 << 30) + 8, host_only=True).graph
    _refused(g.tree_verify, *VERIFY.values(), match="vocab", status=M.MPK_ERR_UNSUPPORTED)
    _refused(g.tree_append, *APPEND.values(), match="host_only")   # (looks at no logits)


def test_no_rows_need_no_buffers():
    g = RowsModel(host_only=True).graph
    for call, args, none in ((g.tree_append, APPEND, ("parents", "qkv", "stride", "q", "q_stride")),
                             (g.tree_attend, ATTEND, ("parents", "q", "q_stride", "out", "out_stride", "work")),
                             (g.tree_verify, VERIFY, ("parents", "tokens", "logits", "stride", "draft", "draft_stride", "uniforms", "path", "logprobs", "work")),
                             (g.tree_keep, KEEP, ("lengths", "path"))):
        empty = dict(args, n_rows=0, **dict.fromkeys(none, 0))
        assert list(empty) == list(args)
        _refused(call, *empty.values(), match="host_only")
        _refused(call, *dict(empty, n_rows=1).values(), match="NULL")
        _refused(call, *dict(empty, n_seqs=0).values(), match="n_seqs")


def test_a_cache_too_long_for_the_cuts():
    g = RowsModel(max_seq=(1 << 28) + 8, batch=1, host_only=True).graph
    for call, args in ((g.tree_append, APPEND), (g.tree_attend, ATTEND), (g.tree_keep, KEEP)):
        _refused(call, *args.values(), match="max_seq", status=M.MPK_ERR_UNSUPPORTED)
    _refused(g.tree_verify, *VERIFY.values(), match="host_only")   # (looks at no cache)


def test_a_serving_graph_and_a_task_dag():
    g, dag = RowsModel(page=16, pages=99, serving=1, greedy_loop=1, host_only=True).graph, M.compile_dag(2, [(0, 1)])
    for name, args in (("tree_append", APPEND), ("tree_attend", ATTEND), ("tree_verify", VERIFY), ("tree_keep", KEEP)):
        _refused(getattr(g, name), *args.values(), match="server")
        _refused(getattr(dag, name), *args.values(), match="DAG")


def test_constants():
    text = open(M.binding.__file__.replace("paper_2512_22219_amd/binding.py", "include/mpk.h")).read()
    assert "#define MPK_TREE_MAX_NODES 256u" in text and M.TREE_MAX_NODES == 256
    assert "#define MPK_TREE_DRAWN_ONCE 1u" in text and M.TREE_DRAWN_ONCE == 1


def test_results_of_no_rows_on_what_is_read(model):
    """Lengths and next tokens are written for calls of no rows too."""
    far = dict(VERIFY, n_rows=0, **{n: P + 4096 * (i + 9) for i, n in enumerate(("begin", "temperatures", "uniforms", "lengths", "next"))})
    _refused(model.graph.tree_verify, *far.values(), match="host_only")
    _refused(model.graph.tree_verify, *dict(far, next=far["lengths"]).values(), match="next_tokens is lengths")
    for name, says in (("lengths", "lengths"), ("next", "next_tokens")):
        _refused(model.graph.tree_verify, *dict(far, **{name: far["begin"]}).values(), match=f"{says} is row_begin")
        _refused(model.graph.tree_verify, *dict(far, **{name: far["temperatures"]}).values(), match=f"{says} is temperatures")
        _refused(model.graph.tree_verify, *dict(far, **{name: far["uniforms"]}).values(), match="host_only")   # (not looked at)
    _refused(model.graph.tree_verify, *dict(far, path=far["lengths"], logprobs=far["lengths"]).values(), match="host_only")


@pytest.mark.parametrize("rows", [0, 7])
@pytest.mark.parametrize("result", ["lengths", "path", "next", "logprobs"])
def test_results_that_begin_or_end_inside_a_list(model, result, rows):
    says = dict(begin="row_begin", next="next_tokens")
    count = dict(begin=4, parents=rows, tokens=rows, temperatures=3, uniforms=rows, lengths=3, path=rows, next=3, logprobs=rows)
    far = dict(VERIFY, n_seqs=3, n_rows=rows, **{n: P + 65536 * (i + 1) for i, n in enumerate(VERIFY) if VERIFY[n] >= P})
    for on, n in count.items():
        if on == result:
            continue
        name, other = says.get(result, result), says.get(on, on)
        both = f"({name} overlaps {other}|{other} overlaps {name})" if n and count[result] else "host_only"
        for off in (4, 4 * (n - 1), -4, -4 * (count[result] - 1)):
            if off:
                _refused(model.graph.tree_verify, *dict(far, **{result: far[on] + off}).values(), match=both)
        for off in (4 * n, -4 * count[result]):   # side by side
            if off:
                _refused(model.graph.tree_verify, *dict(far, **{result: far[on] + off}).values(), match="host_only")


def test_new_positions_that_begin_or_end_inside_a_list(model):
    says = dict(begin="row_begin")
    far = dict(KEEP, n_seqs=3, n_rows=7, slots=P, **{n: P + 65536 * (i + 1) for i, n in enumerate(KEEP) if KEEP[n] >= P})
    far["slots"] = P + 65536 * 20
    for on, n in dict(begin=4, slots=3, positions=3, lengths=3, path=7).items():
        for off in (4, 4 * (n - 1), -4, -8):
            _refused(model.graph.tree_keep, *dict(far, out=far[on] + off).values(), match=f"positions_out overlaps {says.get(on, on)}")
        for off in (4 * n, -12):
            _refused(model.graph.tree_keep, *dict(far, out=far[on] + off).values(), match="host_only")
