"""easyspec_sample_workspace_bytes: a workspace sized for the most rows and words holds every smaller call.  Host arithmetic."""
import paper_2502_02493_amd as es

ROWS = (1, 2, 16, 96, 1023, 1024, 1025, 5000, 65535)
VOCABS = (1, 1000, 4096, 4097, 8192, 8193, 50257, 152064, 1 << 20)


def test_fewer_rows_or_words_never_need_more():
    for a in range(len(ROWS)):
        for b in range(len(VOCABS)):
            need = es.easyspec_sample_workspace_bytes(ROWS[a], VOCABS[b])
            assert need > 0
            for i in range(a + 1):
                for j in range(b + 1):
                    assert es.easyspec_sample_workspace_bytes(ROWS[i], VOCABS[j]) <= need, (ROWS[i], VOCABS[j], ROWS[a], VOCABS[b])


def test_short_rows_need_next_to_nothing():
    assert es.easyspec_sample_workspace_bytes(65535, 8192) == 16
