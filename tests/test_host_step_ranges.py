"""Launches and refusals of the operators of a generation step at the ends of their ranges, on the host.  No GPU."""
from test_host_steps import encode  # noqa: F401 (a fixture)


def test_the_workspace_of_attention_does_not_grow_with_the_rows_of_prompts(encode):  # noqa: F811
    # an 8-bit cache's page is 32 KB a key head of 256: a workspace of a few hundred MB is a few long streams'
    asked = [(rows, seqs, heads, kv, dim, dtype, 256) for dim in (64, 128, 256) for dtype in (0, 1) for kv, heads in ((1, 1), (1, 16), (8, 8), (8, 64), (96, 96))
             for seqs in (1, 3, 32) for rows in (1, 100, 2048, 8192, 65536, 262144) if rows >= seqs]
    for a, p in zip(asked, encode([("attend",) + x for x in asked])):
        assert not isinstance(p, str), (a, p)
        assert p[4] <= 600 << 20, (a, p[4] >> 20)
        if a[1] == 1:  # one sequence: units of no more tiles than go at once
            assert p[4] <= 80 << 20, (a, p[4] >> 20)
