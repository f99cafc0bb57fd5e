"""Further calls that the entry points of the paged cache refuse, on the host, before anything touches a device."""
from paper_2406_18139_b200 import binding as B
from tests.test_paged_abi import FAKE, append, paged

MORE = FAKE + (1 << 30)                         # another aligned address


def test_queries_in_place_have_one_set_of_strides():
    wide = lambda tok, head: B.Layout(8, 2, 128, tok, head, 2 * 128, 128, 0.0)
    ws = dict(ws_bytes=0)                       # (nothing may run)
    assert append(layout=wide(8 * 128, 128), q=FAKE, q_out=FAKE, **ws) == B.ERR_WORKSPACE_TOO_SMALL
    assert append(layout=wide(12 * 128, 128), q=FAKE, q_out=FAKE, **ws) == B.ERR_INVALID_ARG
    assert append(layout=wide(8 * 128, 256), q=FAKE, q_out=FAKE, **ws) == B.ERR_INVALID_ARG
    assert append(paged(q_stride_tok=2048), q=FAKE, q_out=FAKE, **ws) == B.ERR_INVALID_ARG
    # elsewhere they may differ, and so may the token's stride of a single token, the head's of a single head
    assert append(layout=wide(12 * 128, 256), q=FAKE, q_out=MORE, **ws) == B.ERR_WORKSPACE_TOO_SMALL
    assert append(layout=wide(12 * 128, 128), cu=(0, 1), q=FAKE, q_out=FAKE, **ws) == B.ERR_WORKSPACE_TOO_SMALL
    assert append(paged(hq=1, hkv=1, q_stride_head=512), layout=B.Layout(1, 1, 128, 128, 128, 128, 128, 0.0), q=FAKE, q_out=FAKE,
                  **ws) == B.ERR_WORKSPACE_TOO_SMALL
