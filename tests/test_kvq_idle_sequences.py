"""Sequences that a call on caches held in 4 bits leaves alone: what stands in their entries of the other host arrays is not looked at."""
import pytest

import paper_2502_02493_amd as es
from test_kvq_refusals import attend, layout, load, no_memory, refused, select, store

ANY = [-1, 2 ** 31 - 1, -2 ** 31, 97]


@pytest.mark.parametrize("value", ANY)
def test_entries_of_a_sequence_without_slots(value):
    for name in ("src_from", "to", "lens"):
        change = {"src_from": [0, 0, 39, 5], "to": [0, 7, 60, 86], "lens": [96, 96, 61, 96]}[name]
        no_memory(store(**{name: [change[0], value, *change[2:]]}))
        refused(store(**{name: [change[0], value, *change[2:]], "n_slots": [40, 1, 1, 10]}))        # with slots of its own it counts
    for name, change in (("from_", [0, 0, 95, 5]), ("to", [0, 7, 39, 30])):
        no_memory(load(**{name: [change[0], value, *change[2:]]}))
        refused(load(**{name: [change[0], value, *change[2:]], "n_slots": [40, 1, 1, 10]}))


@pytest.mark.parametrize("value", ANY)
def test_lens_of_a_sequence_without_tokens(value):
    for call in (attend, select):
        no_memory(call(lens=[1, 96, value, 20]))
        refused(call(lens=[1, 96, value, 20], n_tokens=[1, 6, 1, 16]))
    assert es.easyspec_kvq_attention_workspace_bytes(layout(), [1, 6, 0, 16], [1, 96, value, 20], 4, 0) == 0
    assert es.easyspec_kvq_select_workspace_bytes(layout(), [1, 6, 0, 16], [1, 96, value, 20], 4, 4) > 0
