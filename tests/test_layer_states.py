"""pced_summarize between pced_append and pced_attend, without a GPU: a call that has nothing to do, or brings
other layers up to date, takes nothing back (stand-ins of tests/layer_path.cpp)."""
from tests.test_layer_path import OK, STATE, Layers, layer_host  # noqa: F401

FEW = (3, 1, 1)


def _covers(b):
    return [r[4] for r in b.calls("append_rows")]


def test_summarize_keeps_what_appends_have_summarised(layer_host):  # noqa: F811
    b = Layers(layer_host, [30, 200], 200, n_layers=2)
    assert b.bind() == OK and b.summarize() == OK
    assert b.append(n=20) == OK and _covers(b) == [1] and b.attend(n=20, sel=FEW) == OK
    assert b.summarize() == OK and b.attend(n=20, sel=FEW) == OK
    assert b.summarize() == OK and b.advance(20) == OK
    assert b.append(n=20) == OK and _covers(b) == [1] and b.attend(n=20, sel=FEW) == OK
    assert b.summarize() == OK and b.advance(3) == OK and b.append() == OK and b.attend(sel=FEW) == OK


def test_summarize_of_layers_in_different_states(layer_host):  # noqa: F811
    b = Layers(layer_host, [30, 200], 200, n_layers=2)
    assert b.append(layer=1, layers=1, n=5) == OK and b.bind() == OK and b.summarize() == OK
    assert b.append(layers=1, n=5) == OK and _covers(b) == [1]
    # layer 1's rows came before the summaries were up to date: they stay unsummarised until the lengths take them in
    assert b.summarize() == OK
    assert b.attend(layers=1, n=5, sel=FEW) == OK and b.attend(layer=1, layers=1, n=5, sel=FEW) == STATE
    assert b.advance(5) == OK
    assert b.append(layers=1) == OK and _covers(b) == [1] and b.append(layer=1, layers=1) == OK and _covers(b) == [0]
    assert b.attend(layers=1, sel=FEW) == OK and b.attend(layer=1, layers=1, sel=FEW) == STATE
    assert b.summarize() == OK and b.calls("summarize")[0][1] == 5
    assert b.attend(layers=1, sel=FEW) == OK and b.attend(layer=1, layers=1, sel=FEW) == STATE
    assert b.append(layer=1, layers=1) == OK and _covers(b) == [1] and b.attend(sel=FEW) == OK


def test_a_new_buffer_and_new_caches_start_over(layer_host):  # noqa: F811
    b = Layers(layer_host, [30, 200], 200, n_layers=2)
    assert b.bind() == OK and b.summarize() == OK and b.append() == OK and b.bind() == OK and b.summarize() == OK
    assert b.attend(sel=FEW) == STATE and b.append() == OK and b.attend(sel=FEW) == OK
    assert b.load(200) == OK and b.summarize() == OK and b.attend(sel=FEW) == STATE
    assert b.append() == OK and b.attend(sel=FEW) == OK
    assert b.step() == OK and b.summarize() == OK and b.attend(sel=FEW) == STATE   # (nothing appended)
