"""sync_attn_status without a GPU."""


def test_null_plan():
    from paper_2608_13757_gb300 import build
    build.build()
    import paper_2608_13757_gb300 as sg
    assert sg.lib().sync_attn_status(None) == sg.ERR_ARG
    assert "NULL" in sg.lib().sync_last_error().decode()
